"""Kept states of more than 2^31 elements: what sums over the whole of a long sequence, and the rows along it."""
import torch

import pytest

import paper_1801_04380_amd as sn
from test_gpu_seq import close, f64

pytestmark = pytest.mark.gpu


def recur(a, b):
    """h[t] = a[t] h[t-1] + b[t] along the rows, by doubling."""
    k = 1
    while k < len(a):
        b = torch.cat((b[:k], torch.addcmul(b[k:], a[k:], b[:-k])))
        a = torch.cat((a[:k], a[k:] * a[:-k]))
        k *= 2
    return b


def test_long_sequence_with_kept_states_past_32_bits():
    """2048 channels of 64 states: the first, one in the middle and the last channel against the same scan in 64 bits, all rows of them and
    their gradients of A, D and dt_bias; the states before every 16th token are read where their offsets are largest."""
    D, N = 2048, 64
    rows = (1 << 31) // (D * N) * 16 + 96
    g = torch.Generator(device="cuda").manual_seed(21)
    r = lambda n, m: torch.rand(n, m, generator=g, device="cuda") + 0.5  # noqa: E731
    u, dt, B, C, z, dy = r(rows, D), r(rows, D) - 2.0, r(rows, N), r(rows, N), r(rows, D), r(rows, D)
    A, skip, bias = -(torch.arange(1, N + 1, device="cuda") / 16 + r(D, 1)), r(D, 1)[:, 0].contiguous(), r(D, 1)[:, 0].contiguous()
    shape = sn.scan_shape(rows, D, N, 1, 1, sn.SN_F32, False)
    states = torch.empty(sn.sn_scan_states_bytes(shape), dtype=torch.uint8, device="cuda")
    assert states.numel() > 4 << 31
    ws = torch.empty(max(sn.sn_scan_workspace_query(shape, i)[1] for i in (sn.SN_SCAN_FWD, sn.SN_SCAN_BWD)), dtype=torch.uint8, device="cuda")
    y, du, ddt, dz, dA, dD, db = (torch.empty_like(t) for t in (u, u, u, u, A, skip, bias))
    dB, dC, hT = torch.empty_like(B), torch.empty_like(C), torch.empty(1, D, N, device="cuda")
    args = (u, dt, A, B, C, skip, z, bias)
    sn.sn_scan_fwd(*args, y, hT=hT, states=states, workspace=ws)
    sn.sn_scan_bwd(*args, dy, du, ddt, dA, dB, dC, dD, dz, db, ws, states=states)
    del states, ws, dB, dC
    for c in (0, 1023, D - 1):
        cu, cdt, cz, cdy = (t[:, c].double() for t in (u, dt, z, dy))
        raw = cdt + bias[c].double()
        delta, sig, rate = torch.nn.functional.softplus(raw, threshold=50.0), torch.sigmoid(cz), A[c].double()
        a, in_ = torch.exp(delta[:, None] * rate), (delta * cu)[:, None] * B.double()
        h = recur(a, in_)
        v = (h * C.double()).sum(1) + skip[c].double() * cu
        gy = cdy * cz * sig
        after = torch.cat((a[1:], torch.zeros_like(a[:1])))
        grad = recur(after.flip(0), (gy[:, None] * C.double()).flip(0)).flip(0)
        q = grad * a * torch.cat((torch.zeros_like(h[:1]), h[:-1]))
        gB = (grad * B.double()).sum(1)
        cddt = (cu * gB + (q * rate).sum(1)) * torch.sigmoid(raw)
        for got, want in ((y[:, c], v * cz * sig), (du[:, c], delta * gB + gy * skip[c].double()), (ddt[:, c], cddt), (dz[:, c], cdy * v * sig * (1 + cz * (1 - sig))),
                          (hT[0, c], h[-1]), (dA[c], (q * delta[:, None]).sum(0)), (dD[c:c + 1], (gy * cu).sum()[None]), (db[c:c + 1], cddt.sum()[None])):
            close(got, f64(want))
