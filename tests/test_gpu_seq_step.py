"""Single tokens of the scan where a state must neither move nor become undefined: delta = 0, and rates at the ends of their range."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
from oracle import seq_oracle as oracle
from test_gpu_seq import SENTINEL, bytes_, close

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rates", [[1.0, -INF, 0.0, -1.0], [-INF] * 5, [-1.0, -INF, -3.402823466e38] + [-INF] * 14])
@pytest.mark.parametrize("softplus", [False, True])
def test_step_does_what_the_forward_does(dtype, rates, softplus):
    """Tokens with delta = 0 (dt = 0, or so far below zero that its softplus is) among others: a state is kept as it is by the former, and one
    whose rate is -inf is only what came in last after the latter.  Both calls form the same decay, once from the states of a
    sequence and once token by token; all values here are whole or powers of two but for the decays of rate 1 and -1."""
    D, N, L = 6, len(rates), 5
    still = -300.0 if softplus else 0.0
    dt = torch.tensor([still, still, 2.0, still, 1.0])[:, None].expand(L, D).contiguous().to(dtype).cuda()
    u, B, C = torch.ones(L, D, device="cuda", dtype=dtype), torch.ones(L, N, device="cuda", dtype=dtype), torch.ones(L, N, device="cuda", dtype=dtype)
    A = torch.tensor(rates, device="cuda").repeat(D, 1)
    h0 = torch.full((1, D, N), 4.0, device="cuda")
    y, hT = torch.full((L, D), SENTINEL, device="cuda", dtype=dtype), torch.full((1, D, N), SENTINEL, device="cuda")
    sn.sn_scan_fwd(u, dt, A, B, C, None, None, None, y, h0=h0, hT=hT, softplus=softplus)
    state, out = h0.clone(), torch.full((L, D), SENTINEL, device="cuda", dtype=dtype)
    for t in range(L):
        sn.sn_scan_step(u[t:t + 1], dt[t:t + 1], A, B[t:t + 1], C[t:t + 1], None, None, None, out[t:t + 1], state, softplus=softplus)
        if t < 2:
            assert (state == 4).all(), t
    d = [0.0, 0.0, np.log1p(np.exp(2.0)) if softplus else 2.0, 0.0, np.log1p(np.exp(1.0)) if softplus else 1.0]
    want = np.full((L, N), 4.0)
    for t, delta in enumerate(d):
        want[t] = (np.exp(delta * np.maximum(rates, -1e30)) if delta else 1.0) * want[max(t - 1, 0)] + delta
    for got in (y, out):
        close(got, want.sum(1)[:, None].repeat(D, 1), dtype)
    for got in (hT, state):
        close(got, want[None, -1:].repeat(D, 1))


def test_backward_of_states_that_vanish_at_once():
    """A = -inf and delta > 0: nothing is kept, so gradients are those of rows on their own, and none reaches A."""
    rows, D, N = 50, 6, 4
    g = torch.Generator().manual_seed(1)
    u, dy, B, C = (torch.randn(rows, n, generator=g) for n in (D, D, N, N))
    dt = torch.rand(rows, D, generator=g) + 0.5
    A = torch.full((D, N), -INF)
    c = [t.cuda() for t in (u, dt, A, B, C)]
    new = [torch.full_like(t, SENTINEL) for t in c]
    du, ddt, dA, dB, dC = new
    shape = sn.scan_shape(rows, D, N, 1, 1, sn.SN_F32, False, False)
    ws = bytes_(sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD)[1] + sn.sn_scan_states_bytes(shape))
    sn.sn_scan_bwd(*c, None, None, None, dy.cuda(), du, ddt, dA, dB, dC, None, None, None, ws, softplus=False)
    f = [t.double().numpy() for t in (u, dt, torch.full((D, N), -1e30), B, C)]
    want = oracle.scan_bwd(*f, None, None, None, dy.double().numpy(), [rows], softplus=False)
    assert (dA == 0).all()
    for got, k in ((du, "du"), (ddt, "ddt"), (dB, "dB"), (dC, "dC")):
        close(got, want[k])
