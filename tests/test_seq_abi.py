"""CPU checks of the C ABI of the token-sequence layers: symbols, what is refused before anything is launched, workspace queries."""
import ctypes
import os
import re

import pytest
import torch

import paper_1801_04380_amd as sn
from paper_1801_04380_amd import _lib, seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, BAD, UNSUPPORTED, SMALL = 0, 1, 2, 3
P = [ctypes.c_void_p((i + 1) << 20) for i in range(40)]   # aligned addresses a MiB apart, never read here


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sn_seq.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sn_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(seq.SIGNATURES) and len(names) == 12
    for n in names:
        assert hasattr(_lib.load(), n) and n in sn.__all__


def conv(call, n, **kw):
    """status of a call with valid arguments but for those in kw: p<i> a pointer, anything else a field of the shape or an argument."""
    s = seq.Conv1dShape(64, 4, 32, 4, 1, sn.SN_BF16, 32, 32, 32)
    return _run(call, s, n, kw)


def _run(call, s, n, kw):
    p, extra = list(P[:n]), {}
    for k, v in kw.items():
        if re.fullmatch(r"p\d+", k):
            p[int(k[1:])] = v
        elif hasattr(s, k):
            setattr(s, k, v)
        else:
            extra[k] = v
    return call(p, s, **extra)


def _fwd(p, s):
    return seq._fn("sn_causal_conv1d_fwd")(*p[:4], ctypes.byref(s), *p[4:7], None)


def _bwd(p, s, bytes_=1 << 30):
    return seq._fn("sn_causal_conv1d_bwd")(*p[:7], ctypes.byref(s), *p[7:12], bytes_, None)


def _step(p, s, num=64):
    return seq._fn("sn_causal_conv1d_step")(*p[:7], num, ctypes.byref(s), None)


SAME = P[0]


@pytest.mark.parametrize("kw,want", [
    (dict(p0=None), BAD), (dict(p1=None), BAD), (dict(p3=None), BAD), (dict(p0=ctypes.c_void_p(4097)), BAD), (dict(p2=ctypes.c_void_p(4098)), BAD), (dict(p3=SAME), BAD),
    (dict(channels=0), BAD), (dict(width=0), BAD), (dict(width=9), UNSUPPORTED), (dict(dtype=2), BAD), (dict(silu=2), BAD), (dict(rows=-1), BAD), (dict(ld_x=31), BAD),
    (dict(ld_y=16), BAD), (dict(rows=1 << 32), UNSUPPORTED), (dict(channels=1 << 30, ld_x=1 << 30, ld_y=1 << 30, ld_dx=1 << 30), UNSUPPORTED),
])
def test_conv1d_refusals(kw, want):
    assert conv(_fwd, 7, **kw) == want
    assert conv(_bwd, 12, **kw) == want
    assert conv(_step, 7, **kw) == want


def test_conv1d_refusals_of_one_call():
    assert conv(_fwd, 7, p4=None, rows=63) == BAD                       # equal lengths: seqs divides rows
    assert conv(_fwd, 7, seqs=0) == BAD
    assert conv(_fwd, 7, p5=P[6]) == BAD                                # state_in is state_out
    assert conv(_fwd, 7, rows=0, p0=None, p3=None, p5=None, p6=None) == OK
    assert conv(_bwd, 12, p4=P[0]) == BAD and conv(_bwd, 12, p4=P[3]) == BAD and conv(_bwd, 12, p4=None) == BAD
    assert conv(_bwd, 12, p5=None) == BAD and conv(_bwd, 12, p11=None) == BAD and conv(_bwd, 12, p11=ctypes.c_void_p(4096 + 128)) == BAD
    assert conv(_bwd, 12, p9=P[10]) == BAD and conv(_bwd, 12, ld_dx=31) == BAD
    need = sn.sn_causal_conv1d_scratch_bytes(64, 32, 4)
    assert need > 0 and need % 256 == 0 and conv(_bwd, 12, bytes_=need - 1) == SMALL
    assert conv(_step, 7, num=-1) == BAD and conv(_step, 7, p4=None) == BAD and conv(_step, 7, p6=None, num=63) == BAD
    assert conv(_step, 7, p6=ctypes.c_void_p(4098)) == BAD and conv(_step, 7, rows=0) == OK
    assert sn.sn_causal_conv1d_scratch_bytes(64, 32, 9) == 0 and sn.sn_causal_conv1d_scratch_bytes(-1, 32, 4) == 0 and sn.sn_causal_conv1d_scratch_bytes(0, 32, 4) > 0


def heads(call, **kw):
    s = seq.HeadnormShape(64, 4, 2, 16, 16, 0, sn.SN_F32, 1e-6, 64, 32, 64, 32, 64, 32)
    return _run(call, s, 14, kw)


def _hfwd(p, s):
    return seq._fn("sn_headnorm_rot_fwd")(*p[:8], ctypes.byref(s), None)


def _hbwd(p, s, bytes_=1 << 30):
    return seq._fn("sn_headnorm_rot_bwd")(*p[:12], ctypes.byref(s), p[12], bytes_, None)


@pytest.mark.parametrize("kw,want", [
    (dict(p0=None), BAD), (dict(p1=None), BAD), (dict(p5=None), BAD), (dict(p6=None), BAD), (dict(p7=None), BAD), (dict(p1=ctypes.c_void_p(4098)), BAD),
    (dict(p4=ctypes.c_void_p(4097)), BAD), (dict(head_dim=15), BAD), (dict(rot_dim=18), BAD), (dict(rot_dim=3), BAD), (dict(q_heads=0), BAD), (dict(k_heads=-1), BAD),
    (dict(eps=0.0), BAD), (dict(eps=float("nan")), BAD), (dict(interleaved=3), BAD), (dict(dtype=7), BAD), (dict(ld_q=63), BAD), (dict(ld_yk=31), BAD), (dict(rows=-1), BAD),
    (dict(head_dim=514, ld_q=1 << 20, ld_k=1 << 20, ld_yq=1 << 20, ld_yk=1 << 20), UNSUPPORTED), (dict(rows=1 << 32), UNSUPPORTED), (dict(p6=SAME, ld_yq=128), BAD),
])
def test_headnorm_refusals(kw, want):
    assert heads(_hfwd, **kw) == want
    if "p6" not in kw or kw["p6"] is None:
        assert heads(_hbwd, **kw) == want


def test_headnorm_refusals_of_one_call():
    assert heads(_hfwd, rows=0, p0=None, p1=None, p6=None, p7=None) == OK
    assert heads(_hbwd, p8=P[0]) == BAD and heads(_hbwd, p9=P[1]) == BAD and heads(_hbwd, p8=None) == BAD and heads(_hbwd, p8=P[6], ld_dq=96) == BAD
    assert heads(_hbwd, p12=None) == BAD
    need = sn.sn_headnorm_rot_scratch_bytes(64, 4, 2, 16)
    assert need > 0 and heads(_hbwd, bytes_=need - 1) == SMALL and sn.sn_headnorm_rot_scratch_bytes(64, 4, 2, 514) == 0


def scan(call, n, **kw):
    s = sn.scan_shape(64, 32, 16, 2, 4, sn.SN_BF16, True)
    for f in ("u", "dt", "b", "c", "z", "y", "du", "ddt", "db", "dc", "dz"):
        setattr(s, "ld_" + f, 32)
    return _run(call, s, n, kw)


def _sfwd(p, s, bytes_=1 << 20):
    return seq._fn("sn_scan_fwd")(*p[:9], ctypes.byref(s), *p[9:14], bytes_, None)


def _sbwd(p, s, bytes_=1 << 40):
    return seq._fn("sn_scan_bwd")(*p[:17], ctypes.byref(s), *p[17:23], bytes_, None)


def _sstep(p, s, num=64):
    return seq._fn("sn_scan_step")(*p[:12], num, ctypes.byref(s), None)


@pytest.mark.parametrize("kw,want", [
    (dict(p0=None), BAD), (dict(p2=None), BAD), (dict(p4=None), BAD), (dict(p8=None), BAD), (dict(p1=ctypes.c_void_p(4097)), BAD), (dict(p5=ctypes.c_void_p(4098)), BAD),
    (dict(channels=0), BAD), (dict(states=0), BAD), (dict(groups=3), BAD), (dict(groups=0), BAD), (dict(dtype=2), BAD), (dict(softplus=2), BAD), (dict(rows=-1), BAD),
    (dict(states=65, ld_b=1000, ld_c=1000), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(ld_u=31), BAD), (dict(ld_b=31), BAD), (dict(ld_c=31), BAD),
    (dict(ld_z=31), BAD), (dict(ld_y=31), BAD),
])
def test_scan_refusals(kw, want):
    assert scan(_sfwd, 14, **kw) == want
    assert scan(_sbwd, 23, **kw) == want
    assert scan(_sstep, 12, **kw) == want


def test_scan_refusals_of_one_call():
    assert scan(_sfwd, 14, p8=P[0]) == BAD and scan(_sfwd, 14, p11=P[10]) == BAD and scan(_sfwd, 14, p9=None) == BAD and scan(_sfwd, 14, ragged=0) == BAD
    assert scan(_sfwd, 14, p13=None) == BAD and scan(_sfwd, 14, p13=ctypes.c_void_p(4096 + 64)) == BAD and scan(_sfwd, 14, seqs=0) == BAD
    assert scan(_sfwd, 14, p9=None, ragged=0, rows=63) == BAD
    assert scan(_sfwd, 14, rows=0, p0=None, p1=None, p3=None, p4=None, p8=None, p11=None) == OK
    for i in (9, 10, 11, 12, 13, 14, 15, 16):                              # du ddt dA dB dC dD dz ddt_bias
        assert scan(_sbwd, 23, **{"p%d" % i: None}) == BAD, i
    assert scan(_sbwd, 23, p5=None) == BAD and scan(_sbwd, 23, p6=None) == BAD and scan(_sbwd, 23, p7=None) == BAD   # a gradient of what is not there
    assert scan(_sbwd, 23, p9=P[0]) == BAD and scan(_sbwd, 23, p9=P[10]) == BAD and scan(_sbwd, 23, p21=P[20]) == BAD and scan(_sbwd, 23, p22=None) == BAD
    assert scan(_sbwd, 23, ld_du=31) == BAD and scan(_sbwd, 23, ld_dz=31) == BAD
    s = sn.scan_shape(64, 32, 16, 2, 4, sn.SN_BF16, True)
    mn, pf = sn.sn_scan_workspace_query(s, sn.SN_SCAN_BWD)
    assert 0 < mn <= pf and mn % 256 == 0
    assert scan(_sbwd, 23, bytes_=mn - 1) == SMALL
    assert scan(_sbwd, 23, bytes_=mn + sn.sn_scan_states_bytes(s) - 1, p19=None) == SMALL
    assert scan(_sstep, 12, num=-1) == BAD and scan(_sstep, 12, p9=None) == BAD and scan(_sstep, 12, p11=None, num=63) == BAD and scan(_sstep, 12, rows=0) == OK
    with pytest.raises(sn.SnError):
        sn.sn_scan_workspace_query(sn.scan_shape(64, 32, 65), sn.SN_SCAN_FWD)
    assert sn.sn_scan_states_bytes(sn.scan_shape(64, 32, 65)) == 0


def test_scan_workspace_grows_with_the_tokens_where_channels_are_few():
    wide, narrow = sn.scan_shape(32 * 512, 4096, 16, seqs=32), sn.scan_shape(32768, 64, 16)
    assert sn.sn_scan_workspace_query(wide, sn.SN_SCAN_FWD) == (0, 0)
    assert sn.sn_scan_workspace_query(narrow, sn.SN_SCAN_FWD)[1] > 0
    # the state before every 16th token
    assert sn.sn_scan_states_bytes(wide) == 16384 // 16 * 4096 * 16 * 4
    assert sn.sn_scan_states_bytes(sn.scan_shape(34, 64, 16, seqs=2)) == 4 * 64 * 16 * 4


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="current device"):
        sn.sn_causal_conv1d_fwd(x, torch.zeros(8, 4), None, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="current device"):
        sn.sn_headnorm_rot_fwd(x, None, None, None, None, None, torch.zeros(4, 8), None, 8)
    with pytest.raises(ValueError, match="whole heads"):
        sn.sn_headnorm_rot_fwd(x, None, None, None, None, None, torch.zeros(4, 8), None, 3)
    with pytest.raises(ValueError, match="whole groups"):
        sn.sn_scan_fwd(x, x, torch.zeros(8, 3), x, x, None, None, None, torch.zeros(4, 8))


def test_kept_states_are_aligned():
    P8 = ctypes.c_void_p(P[12].value + 8)
    assert scan(_sfwd, 14, p12=P8) == BAD and scan(_sbwd, 23, p19=ctypes.c_void_p(P[19].value + 16)) == BAD


@pytest.mark.parametrize("field", ["u", "dt", "b", "c", "z", "y"])
def test_scan_refuses_rows_too_far_apart(field):
    kw = {"ld_" + field: (1 << 24) + 1}
    assert scan(_sfwd, 14, **kw) == UNSUPPORTED and scan(_sbwd, 23, **kw) == UNSUPPORTED and scan(_sstep, 12, **kw) == UNSUPPORTED


@pytest.mark.parametrize("field", ["du", "ddt", "db", "dc", "dz"])
def test_scan_refuses_gradients_rows_too_far_apart(field):
    assert scan(_sbwd, 23, **{"ld_" + field: (1 << 24) + 1}) == UNSUPPORTED


def test_sizes_beyond_the_grids():
    most, rows = 65535, 1 << 30
    big = lambda n: {"ld_" + f: n for f in ("u", "dt", "b", "c", "z", "y", "du", "ddt", "db", "dc", "dz")}  # noqa: E731
    assert scan(_sfwd, 14, rows=rows + 1) == UNSUPPORTED and scan(_sbwd, 23, rows=rows + 1) == UNSUPPORTED
    assert scan(_sfwd, 14, seqs=1 << 24) == UNSUPPORTED and scan(_sbwd, 23, seqs=1 << 24) == UNSUPPORTED
    assert scan(_sfwd, 14, channels=most * 16 + 1, groups=1, **big(1 << 24)) == UNSUPPORTED
    assert scan(_sfwd, 14, channels=40000 * 17, groups=40000, states=1, **big(1 << 24)) == UNSUPPORTED      # two blocks a group
    assert scan(_sstep, 12, rows=1 << 24) == UNSUPPORTED
    assert conv(_fwd, 7, channels=most * 256 + 1, ld_x=1 << 25, ld_y=1 << 25, ld_dx=1 << 25) == UNSUPPORTED
    assert conv(_step, 7, rows=1 << 24) == UNSUPPORTED and conv(_fwd, 7, seqs=1 << 24) == UNSUPPORTED
    assert heads(_hfwd, rows=rows + 1) == UNSUPPORTED
    assert sn.sn_causal_conv1d_scratch_bytes(rows + 1, 4, 4) == 0 == sn.sn_headnorm_rot_scratch_bytes(rows + 1, 1, 0, 16)


def test_short_sequences_of_equal_length_share_tiles():
    together = sn.scan_shape(2048 * 4, 64, 16, seqs=2048)
    assert sn.sn_scan_states_bytes(together) == 2048 * 4 // 16 * 64 * 16 * 4
    assert sn.sn_scan_states_bytes(sn.scan_shape(64 * 4, 64, 16, seqs=64)) == 64 * 64 * 16 * 4      # few: each on its own
    assert sn.sn_scan_states_bytes(sn.scan_shape(64 * 17, 64, 16, seqs=64)) == 64 * 2 * 64 * 16 * 4
