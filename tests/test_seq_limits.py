"""CPU: limits of sizes that the header of the token-sequence layers names, refused before anything is launched."""
import paper_1801_04380_amd as sn
from test_seq_abi import BAD, OK, UNSUPPORTED, _hbwd, _hfwd, _sfwd, heads, scan


def test_heads():
    wide = {"ld_" + f: 1 << 22 for f in ("q", "k", "yq", "yk", "dq", "dk")}
    for call in (_hfwd, _hbwd):
        assert heads(call, q_heads=1 << 20, k_heads=1, head_dim=2, rot_dim=2, **wide) == UNSUPPORTED
        assert heads(call, q_heads=1 << 20, k_heads=0, head_dim=2, rot_dim=2, rows=-1, **wide) == BAD
    assert heads(_hfwd, q_heads=1 << 20, k_heads=0, head_dim=2, rot_dim=2, rows=0, **wide) == OK
    assert sn.sn_headnorm_rot_scratch_bytes(4, 1 << 20, 1, 2) == 0 < sn.sn_headnorm_rot_scratch_bytes(4, 1 << 20, 0, 2)


def test_rows_of_the_scan_as_far_apart_as_may_be():
    """2^24 elements are accepted: the call goes on to what it refuses next, a state that is its own output."""
    kw = {"ld_u": 1 << 24, "ld_dt": 1 << 24, "ld_y": 1 << 24}
    from test_seq_abi import P
    assert scan(_sfwd, 14, p11=P[10], **kw) == BAD and scan(_sfwd, 14, p11=P[10], **dict(kw, ld_u=(1 << 24) + 1)) == UNSUPPORTED
