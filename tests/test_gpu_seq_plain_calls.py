"""Calls with what may be left out left out: no states in or out, slots in order, one of two weights' gradients, a single row of any stride."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
from oracle import seq_oracle as oracle
from test_gpu_seq import SENTINEL, Data, bytes_, close, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 5])
def test_steps_without_slots(dtype, rows):
    d, D, N, W = Data(dtype, rows), 20, 7, 3
    x, w, state = d.normal(rows, D), d.normal(D, W), d.normal(rows + 2, W - 1, D)
    pool, y = state.cuda(), torch.empty(rows, D, dtype=d.dtype, device="cuda")
    sn.sn_causal_conv1d_step(x.cuda(), w.cuda(), None, y, pool)
    want, end = oracle.conv1d_fwd(f64(x), f64(w), None, [1] * rows, f64(state)[:rows])
    close(y, want, d.dtype)
    assert np.array_equal(f64(pool), np.concatenate([end, f64(state)[rows:]]))
    B, C, A, h = d.normal(rows, N), d.normal(rows, N), -d.uniform(0.5, 1.5, D, N), d.normal(rows + 2, D, N, dtype=torch.float32)
    pool = h.cuda()
    sn.sn_scan_step(x.cuda(), x.cuda(), A.cuda(), B.cuda(), C.cuda(), None, None, None, y, pool)
    want, end = oracle.scan_fwd(f64(x), f64(x), f64(A), f64(B), f64(C), None, None, None, [1] * rows, f64(h)[:rows])
    close(y, want, d.dtype)
    close(pool, np.concatenate([end, f64(h)[rows:]]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_weight_gradient_and_positions_counted(dtype):
    d, rows, Dh = Data(dtype, 1), 37, 32
    q, k, dq, dk = d.normal(rows, 3 * Dh), d.normal(rows, Dh), d.normal(rows, 3 * Dh), d.normal(rows, Dh)
    freq = (100.0 ** (-torch.arange(Dh // 2) / (Dh // 2))).float()
    scratch = bytes_(sn.sn_headnorm_rot_scratch_bytes(rows, 3, 1, Dh))
    pos = np.arange(rows)
    for which in (0, 1):
        gq, gk, dw = torch.empty_like(q).cuda(), torch.empty_like(k).cuda(), torch.full((Dh,), SENTINEL, device="cuda")
        sn.sn_headnorm_rot_bwd(q.cuda(), k.cuda(), None, None, None, freq.cuda(), dq.cuda(), dk.cuda(), gq, gk, None if which else dw, dw if which else None, scratch, Dh)
        for got, x, g, mine in ((gq, q, dq, which == 0), (gk, k, dk, which == 1)):
            dx, want = oracle.headnorm_bwd(f64(x), None, pos, f64(freq), f64(g), Dh, 1e-6, False)
            close(got, dx, d.dtype)
            if mine:
                close(dw, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 75])
def test_scan_and_convolution_without_states(dtype, rows):
    """One sequence, nothing before and nothing asked for behind it; of a single row the tensors' strides do not matter."""
    d, D, N, W = Data(dtype, rows), 24, 6, 4
    line = lambda n: d.normal(1, n).expand(1, n) if rows == 1 else d.normal(rows, n)  # noqa: E731
    u, dt, B, C, dy, x = line(D), line(D), line(N), line(N), line(D), line(D)
    A, w = -d.uniform(0.5, 1.5, D, N), d.normal(D, W, scale=0.5)
    far = lambda t: torch.empty(2, 1 << 20, dtype=d.dtype, device="cuda")[:1, :t.shape[1]].copy_(t) if rows == 1 else t.cuda()  # noqa: E731
    c = [far(u), far(dt), A.cuda(), far(B), far(C)]
    y = far(u)
    sn.sn_scan_fwd(*c, None, None, None, y)
    f = [f64(t) for t in (u, dt, A, B, C)]
    close(y, oracle.scan_fwd(*f, None, None, None, [rows])[0], d.dtype)
    du, ddt, dA, dB, dC = far(u), far(dt), torch.empty(D, N, device="cuda"), far(B), far(C)
    shape = sn.scan_shape(rows, D, N, 1, 1, sn.SN_BF16 if dtype == "bf16" else sn.SN_F32)
    ws = bytes_(sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD)[0] + sn.sn_scan_states_bytes(shape))
    sn.sn_scan_bwd(*c, None, None, None, far(dy), du, ddt, dA, dB, dC, None, None, None, ws)
    want = oracle.scan_bwd(*f, None, None, None, f64(dy), [rows])
    for got, k in ((du, "du"), (ddt, "ddt"), (dB, "dB"), (dC, "dC")):
        close(got, want[k], d.dtype)
    close(dA, want["dA"])
    sn.sn_causal_conv1d_fwd(far(x), w.cuda(), None, y)
    close(y, oracle.conv1d_fwd(f64(x), f64(w), None, [rows])[0], d.dtype)
    dw = torch.empty(D, W, device="cuda")
    sn.sn_causal_conv1d_bwd(far(x), w.cuda(), None, far(dy), du, dw, None, bytes_(sn.sn_causal_conv1d_scratch_bytes(rows, D, W)))
    wdx, wdw, _, _ = oracle.conv1d_bwd(f64(x), f64(w), None, f64(dy), [rows])
    close(du, wdx, d.dtype)
    close(dw, wdw)
