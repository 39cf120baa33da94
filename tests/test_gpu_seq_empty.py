"""Batches padded with empty sequences, more of them than there are workgroups to look at them at once."""
import pytest
import torch

import paper_1801_04380_amd as sn
from test_gpu_seq import SENTINEL, bytes_, close, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S,channels", [(70001, 5), (3000, 40)])
@pytest.mark.parametrize("given", [True, False])
def test_states_of_empty_sequences(dtype, S, channels, given):
    """Some sequences among many empty ones: theirs are the states that the same call leaves without the empty ones; the others keep what they were
    given, or zeros."""
    D, N, W = channels, 6, 4
    g = torch.Generator(device="cuda").manual_seed(S)
    lengths = torch.zeros(S, dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 1, 17, 64, 1000, S // 2, S - 2], device="cuda")
    lengths[some] = torch.tensor([3, 1, 20, 2, 5, 33, 9], dtype=torch.int32, device="cuda")
    rows = int(lengths.sum())
    off = lambda n: torch.cat((torch.zeros(1, device="cuda"), n.cumsum(0))).int()  # noqa: E731
    r = lambda *s, t=dtype: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    x, dt, B, C, dy, w, A = r(rows, D), r(rows, D), r(rows, N), r(rows, N), r(rows, D), r(D, W), -torch.rand(D, N, generator=g, device="cuda")
    s0, h0, dhT = r(S, W - 1, D), r(S, D, N, t=torch.float32), r(S, D, N, t=torch.float32)
    found = []
    for pick, n in ((slice(None), S), (some, len(some))):
        kw, new = {"seqs": n, "offsets": off(lengths[pick])}, torch.full_like
        y, yc, du, ddt, dB, dC, dA = new(x, SENTINEL), new(x, SENTINEL), new(x, SENTINEL), new(x, SENTINEL), new(B, SENTINEL), new(C, SENTINEL), new(A, SENTINEL)
        s1, hT, dh0 = new(s0[pick], SENTINEL), new(h0[pick], SENTINEL), new(h0[pick], SENTINEL)
        sn.sn_causal_conv1d_fwd(x, w, None, yc, state_in=s0[pick] if given else None, state_out=s1, **kw)
        sn.sn_scan_fwd(x, dt, A, B, C, None, None, None, y, h0=h0[pick] if given else None, hT=hT, **kw)
        shape = sn.scan_shape(rows, D, N, 1, n, sn.SN_BF16 if dtype == torch.bfloat16 else sn.SN_F32, True)
        ws = bytes_(sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD)[0] + sn.sn_scan_states_bytes(shape))
        sn.sn_scan_bwd(x, dt, A, B, C, None, None, None, dy, du, ddt, dA, dB, dC, None, None, None, ws, h0=h0[pick] if given else None, dhT=dhT[pick] if given else None,
                       dh0=dh0, **kw)
        found.append((yc, s1, y, hT, du, ddt, dB, dC, dA, dh0))
    empty = lengths == 0
    for k, (a, b) in enumerate(zip(*found)):
        if k in (1, 3, 9):
            source = {1: s0, 3: h0, 9: dhT}[k]
            assert torch.equal(a[empty], source[empty] if given else torch.zeros_like(source[empty])), k
            a = a[some]
        if k == 8:
            close(a, f64(b))   # which rows a sum's stretches end at depends on the pieces
        else:
            assert torch.equal(a, b), k
