"""Sums over very many rows: gradients of what all rows share.

The inputs repeat, so that every term is the same and the roundings of a sum all go one way as long as it stays between two powers of two: the
worst that a running sum of n terms can do, n * 2^-24 of it.  Sums run over at most 256 terms before they are added, without
loss, to what was summed before.  The terms' own error is on top: a chain of at most 16 tokens, three roundings each, 48 * 2^-24 for a
state and as much for a gradient."""
import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn
from oracle import seq_oracle as oracle
from test_gpu_seq import SENTINEL, bytes_

pytestmark = pytest.mark.gpu
SUM = 256 * 2.0 ** -24


def off(got, want):
    got = got.double().cpu().numpy()
    return (np.abs(got - want) / np.abs(want)).max()


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("D,N", [(16, 4), (40, 20)])
def test_scan(ragged, cut, D, N):
    """2^16 sequences of the same 16 tokens; with the least workspace one workgroup walks along all of them."""
    S, L = 1 << 16, 16
    g = torch.Generator().manual_seed(D)
    r = lambda *s: torch.rand(*s, generator=g) * 0.5 + 0.5  # noqa: E731
    one = [r(L, D), r(L, D) - 0.5, -r(D, N), r(L, N), r(L, N), r(D), r(L, D), -r(D)]            # u, dt, A, B, C, D, z, dt_bias
    dy, many = r(L, D), lambda t: t.repeat(S, 1).cuda()  # noqa: E731
    u, dt, A, B, C, skip, z, bias = (t.cuda() if i in (2, 5, 7) else many(t) for i, t in enumerate(one))
    want = oracle.scan_bwd(*(t.double().numpy() for t in one), dy.double().numpy(), [L])
    shape = sn.scan_shape(S * L, D, N, 1, S, sn.SN_F32, ragged)
    kw = {"seqs": S, "offsets": (torch.arange(S + 1, dtype=torch.int32) * L).cuda() if ragged else None}
    new = lambda t: torch.full_like(t, SENTINEL)  # noqa: E731
    du, ddt, dA, dB, dC, dD, dz, db = (new(t) for t in (u, dt, A, B, C, skip, z, bias))
    ws = bytes_(sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD)[int(cut)] + sn.sn_scan_states_bytes(shape))
    sn.sn_scan_bwd(u, dt, A, B, C, skip, z, bias, many(dy), du, ddt, dA, dB, dC, dD, dz, db, ws, **kw)
    for got, k in ((dA, "dA"), (dD, "dD"), (db, "ddt_bias")):
        assert off(got, S * want[k]) <= SUM + 96 * 2.0 ** -24, k
    for got, k in ((du, "du"), (dB, "dB"), (dz, "dz")):
        assert off(got[-L:], want[k]) <= 192 * 2.0 ** -24, k


def test_conv1d():
    rows, D, W = 1 << 24, 4, 4
    x, dy, w = torch.full((rows, D), 0.7, device="cuda"), torch.full((rows, D), 0.3, device="cuda"), torch.ones(D, W, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.full((D, W), SENTINEL, device="cuda"), torch.full((D,), SENTINEL, device="cuda")
    sn.sn_causal_conv1d_bwd(x, w, None, dy, dx, dw, db, bytes_(sn.sn_causal_conv1d_scratch_bytes(rows, D, W)), silu=False)
    a, b = float(np.float32(0.7)), float(np.float32(0.3))
    assert off(db, np.full(D, rows * b)) <= SUM
    assert off(dw, np.repeat([(rows - W + 1 + np.arange(W)) * a * b], D, 0)) <= SUM + 2.0 ** -24


def test_headnorm():
    rows, Dh = 1 << 25, 2
    q = torch.tensor([[0.7, -1.3]], device="cuda").repeat(rows, 1)
    dy, k = torch.full((rows, Dh), 0.3, device="cuda"), q[:, :Dh]
    dq, dwq, dwk = torch.empty_like(q), torch.full((Dh,), SENTINEL, device="cuda"), torch.full((Dh,), SENTINEL, device="cuda")
    sn.sn_headnorm_rot_bwd(q, k, None, None, None, None, dy, dy, dq, torch.empty_like(q), dwq, dwk, bytes_(sn.sn_headnorm_rot_scratch_bytes(rows, 1, 1, Dh)), Dh, 1e-6)
    x = q[:1].double().cpu().numpy()
    _, dw = oracle.headnorm_bwd(x, None, np.zeros(1), np.zeros(0), np.full((1, Dh), float(np.float32(0.3))), Dh, 1e-6, False)
    for got in (dwq, dwk):      # a term: the squares' sum, the mean, eps, the root, two products
        assert off(got, rows * dw) <= SUM + 8 * 2.0 ** -24


@pytest.mark.parametrize("big", [float("inf"), 1e38])
def test_sums_past_the_range_are_infinite(big):
    """An infinite term, or terms whose sum is: not NaN, however the rows are cut."""
    rows, D, N = 700, 8, 4
    one, zero, vec = torch.ones(rows, D, device="cuda"), torch.zeros(rows, N, device="cuda"), torch.ones(D, device="cuda")
    dy = torch.full_like(one, big)
    dx, dw, db = torch.empty_like(one), torch.empty(D, 2, device="cuda"), torch.empty(D, device="cuda")
    sn.sn_causal_conv1d_bwd(one, torch.zeros_like(dw), None, dy, dx, dw, db, bytes_(sn.sn_causal_conv1d_scratch_bytes(rows, D, 2)), silu=False)
    # the first tap of the first row is on a zero in front of the sequence, and zero times an infinite dy is none
    assert torch.isposinf(db).all() and torch.isposinf(dw[:, 1]).all() and (torch.isposinf(dw[:, 0]) | (big == float("inf"))).all()
    shape = sn.scan_shape(rows, D, N, 1, 1, sn.SN_F32, False, False)
    for n in sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD):
        A, dD = torch.zeros(D, N, device="cuda"), torch.empty(D, device="cuda")
        sn.sn_scan_bwd(one, one, A, zero, zero, vec, None, None, dy, torch.empty_like(one), torch.empty_like(one), torch.empty_like(A), torch.empty_like(zero),
                       torch.empty_like(zero), dD, None, None, bytes_(n + sn.sn_scan_states_bytes(shape)), softplus=False)
        assert torch.isposinf(dD).all()
    dwq, scratch = torch.empty(2, device="cuda"), bytes_(sn.sn_headnorm_rot_scratch_bytes(rows, 4, 0, 2))
    sn.sn_headnorm_rot_bwd(one, None, None, None, None, None, dy, None, dx, None, dwq, None, scratch, 2)
    assert torch.isposinf(dwq).all()
