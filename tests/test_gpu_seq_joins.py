"""The scan cut into chunks where what happens to a state within a chunk is more than the range of fp32, though the state never leaves it."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
from test_gpu_seq import SENTINEL, bytes_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("N", [4, 20])
def test_a_state_that_crosses_the_range_within_a_chunk(sign, N):
    """24 tokens of delta = 4 multiply a state by e^96 or e^-96, beyond what fp32 holds; all others leave it alone.  From 1e-30 (1e30) on it ends
    at 4.9e11 (2.0e-12), and so does the gradient on its way back.

    Tolerance: log2(e) * A as rounded is off by half a step, 2^-24 of it, so an exponent of 138 by 138 * 2^-24, a factor by ln 2 times that, 5.7e-6.
    Beside it 24 products and exponentials are rounded, each by 2^-23 at most: 2.9e-6.  2e-5 holds both twice over."""
    rows, D = 700, 8
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    dt = z(rows, D)
    dt[40:64] = 4.0
    u, B, C, A = z(rows, D), z(rows, N) + 1, z(rows, N), z(D, N) + sign
    C[-1] = 1.0
    start, end = 10.0 ** (-30 * sign), float(np.exp(96.0 * sign)) * float(np.float32(10.0 ** (-30 * sign)))
    h0 = z(1, D, N) + start
    shape = sn.scan_shape(rows, D, N, 1, 1, sn.SN_F32, False, False)
    cut, whole = sn.sn_scan_workspace_query(shape, sn.SN_SCAN_FWD)[1], 0
    assert cut > whole
    for n in (whole, cut):
        y, hT = z(rows, D) + SENTINEL, z(1, D, N) + SENTINEL
        sn.sn_scan_fwd(u, dt, A, B, C, None, None, None, y, h0=h0, hT=hT, workspace=bytes_(n), softplus=False)
        assert ((hT.double() / end - 1).abs() < 2e-5).all(), n
        assert (y[:-1] == 0).all() and ((y[-1].double() / (N * end) - 1).abs() < 2e-5).all(), n
    least, most = (b + sn.sn_scan_states_bytes(shape) for b in sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD))
    assert most > least
    for n in (least, most):
        du, ddt, dA, dB, dC, dh0 = (torch.full_like(t, SENTINEL) for t in (u, dt, A, B, C, h0))
        sn.sn_scan_bwd(u, dt, A, B, C, None, None, None, z(rows, D), du, ddt, dA, dB, dC, None, None, None, bytes_(n), h0=z(1, D, N), dhT=h0, dh0=dh0,
                       softplus=False)
        assert ((dh0.double() / end - 1).abs() < 2e-5).all(), n
