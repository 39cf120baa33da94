"""The oracle of the token-sequence layers against central differences of its own forward passes, and against closed forms."""
import numpy as np
import pytest

from oracle import seq_oracle as o

RNG = np.random.RandomState(3)


def differences(f, x, step=1e-6):
    """The gradient of the number f(x) by central differences; the error of O(step^2) and of rounding over step are both below 1e-8."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        g[i] = (up - f()) / (2 * step)
        x[i] = keep
    return g


def near(a, b):
    assert np.abs(a - b).max(initial=0) <= 1e-7 * (1 + np.abs(b).max(initial=0))


@pytest.mark.parametrize("silu", [True, False])
def test_conv1d_gradients(silu):
    lengths, D, W = [5, 0, 1, 4], 3, 4
    x, w, b, dy = RNG.randn(10, D), RNG.randn(D, W), RNG.randn(D), RNG.randn(10, D)
    s, ds = RNG.randn(4, W - 1, D), RNG.randn(4, W - 1, D)

    def loss():
        y, end = o.conv1d_fwd(x, w, b, lengths, s, silu)
        return (y * dy).sum() + (end * ds).sum()

    dx, dw, db, dstate = o.conv1d_bwd(x, w, b, dy, lengths, s, ds, silu)
    for got, of in ((dx, x), (dw, w), (db, b), (dstate, s)):
        near(got, differences(loss, of))


def test_conv1d_is_causal_convolution():
    x, w = RNG.randn(6, 1), RNG.randn(1, 3)
    y, end = o.conv1d_fwd(x, w, None, [6], None, False)
    near(y[:, 0], np.convolve(x[:, 0], w[0, ::-1])[:6])
    assert np.array_equal(end[0], x[-2:])


@pytest.mark.parametrize("interleaved", [True, False])
def test_headnorm_gradients(interleaved):
    rows, Dh = 3, 6
    x, w, dy, freq, pos = RNG.randn(rows, 2 * Dh), RNG.randn(Dh), RNG.randn(rows, 2 * Dh), np.array([0.7, 0.1]), np.array([0, 5, 11])
    loss = lambda: (o.headnorm_fwd(x, w, pos, freq, Dh, 0.1, interleaved) * dy).sum()  # noqa: E731
    dx, dw = o.headnorm_bwd(x, w, pos, freq, dy, Dh, 0.1, interleaved)
    near(dx, differences(loss, x))
    near(dw, differences(loss, w))


@pytest.mark.parametrize("gate,softplus,optional", [(True, True, True), (False, True, False), (True, False, True)])
def test_scan_gradients(gate, softplus, optional):
    lengths, E, N, G = [4, 0, 1, 3], 4, 3, 2
    u, B, C, dy = RNG.randn(8, E), RNG.randn(8, G * N), RNG.randn(8, G * N), RNG.randn(8, E)
    dt, A = np.abs(RNG.randn(8, E)) * 0.5, -np.abs(RNG.randn(E, N))
    D, bias = (RNG.randn(E), RNG.randn(E) * 0.1) if optional else (None, None)
    z = RNG.randn(8, E) if gate else None
    h0, dhT = RNG.randn(4, E, N), RNG.randn(4, E, N)

    def loss():
        y, hT = o.scan_fwd(u, dt, A, B, C, D, z, bias, lengths, h0, softplus)
        return (y * dy).sum() + (hT * dhT).sum()

    g = o.scan_bwd(u, dt, A, B, C, D, z, bias, dy, lengths, h0, dhT, softplus)
    of = {"du": u, "ddt": dt, "dA": A, "dB": B, "dC": C, "dh0": h0}
    if optional:
        of.update(dD=D, ddt_bias=bias)
    if gate:
        of["dz"] = z
    for k, v in of.items():
        near(g[k], differences(loss, v))


def test_scan_with_constant_decay_is_a_geometric_sum():
    L, a = 20, 0.8
    y, hT = o.scan_fwd(np.ones((L, 1)), np.ones((L, 1)), np.log([[a]]), np.ones((L, 1)), np.ones((L, 1)), None, None, None, [L], None, False)
    near(y[:, 0], (1 - a ** np.arange(1, L + 1)) / (1 - a))
    near(hT[0, 0], y[-1])
