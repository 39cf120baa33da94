"""The layers along token sequences in 64 bits, token after token, straight from their definitions: numpy only, no code shared
with the library.  Inputs are float64 arrays (of values already rounded to the type that the library gets); `lengths` are the
sequences' rows, packed one behind the other; rows behind the last are in no sequence and come out as NaN."""
import numpy as np


def _sigmoid(x):
    return np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))


def _spans(lengths):
    at = 0
    for s, n in enumerate(lengths):
        yield s, at, at + n
        at += n


def conv1d_fwd(x, w, bias, lengths, state_in=None, silu=True):
    """-> y, state_out"""
    D, W = w.shape
    y, out = np.full_like(x, np.nan), np.zeros((len(lengths), W - 1, D))
    for s, a, b in _spans(lengths):
        line = np.concatenate([np.zeros((W - 1, D)) if state_in is None else state_in[s], x[a:b]])
        for t in range(b - a):
            p = (line[t:t + W] * w.T).sum(0) + (0 if bias is None else bias)
            y[a + t] = p * _sigmoid(p) if silu else p
        out[s] = line[b - a:]
    return y, out


def conv1d_bwd(x, w, bias, dy, lengths, state_in=None, dstate_out=None, silu=True):
    """-> dx, dw, dbias, dstate_in"""
    D, W = w.shape
    dx, dw, db, ds = np.full_like(x, np.nan), np.zeros((D, W)), np.zeros(D), np.zeros((len(lengths), W - 1, D))
    for s, a, b in _spans(lengths):
        line = np.concatenate([np.zeros((W - 1, D)) if state_in is None else state_in[s], x[a:b]])
        g = np.zeros_like(line)
        if dstate_out is not None:
            g[b - a:] += dstate_out[s]
        for t in range(b - a):
            p = (line[t:t + W] * w.T).sum(0) + (0 if bias is None else bias)
            sg = _sigmoid(p)
            dp = dy[a + t] * (sg * (1 + p * (1 - sg)) if silu else 1.0)
            g[t:t + W] += dp * w.T
            dw += (dp * line[t:t + W]).T
            db += dp
        ds[s], dx[a:b] = g[:W - 1], g[W - 1:]
    return dx, dw, db, ds


def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def headnorm_fwd(x, w, positions, inv_freq, head_dim, eps, interleaved):
    """x: (rows, heads * head_dim) -> y"""
    h = x.reshape(x.shape[0], -1, head_dim)
    n = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w)
    y = n.copy()
    one, two = _pairs(2 * len(inv_freq), interleaved)
    angle = (positions.astype(np.float64)[:, None] * inv_freq)[:, None]
    c, s = np.cos(angle), np.sin(angle)
    y[..., one] = n[..., one] * c - n[..., two] * s
    y[..., two] = n[..., two] * c + n[..., one] * s
    return y.reshape(x.shape)


def headnorm_bwd(x, w, positions, inv_freq, dy, head_dim, eps, interleaved):
    """-> dx, dw"""
    h, g = x.reshape(x.shape[0], -1, head_dim), dy.reshape(x.shape[0], -1, head_dim).copy()
    one, two = _pairs(2 * len(inv_freq), interleaved)
    angle = (positions.astype(np.float64)[:, None] * inv_freq)[:, None]
    c, s = np.cos(angle), np.sin(angle)
    g[..., one], g[..., two] = g[..., one] * c + g[..., two] * s, g[..., two] * c - g[..., one] * s
    r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    dw = (g * h * r).sum((0, 1))
    g = g * (1.0 if w is None else w)
    return (r * (g - h * r * r * (g * h).mean(-1, keepdims=True))).reshape(x.shape), dw


def _softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def scan_fwd(u, dt, A, B, C, D, z, bias, lengths, h0=None, softplus=True, states=None):
    """-> y, hT.  states: a list that gets the state before and behind every token, in order."""
    rows, E = u.shape
    N, G = A.shape[1], B.shape[1] // A.shape[1]
    y, hT = np.full_like(u, np.nan), np.zeros((len(lengths), E, N))
    group = np.arange(E) // (E // G)
    for s, a, b in _spans(lengths):
        h = np.zeros((E, N)) if h0 is None else h0[s].copy()
        for t in range(a, b):
            raw = dt[t] + (0 if bias is None else bias)
            delta = _softplus(raw) if softplus else raw
            before = h
            h = np.exp(delta[:, None] * A) * h + (delta * u[t])[:, None] * B[t].reshape(G, N)[group]
            if states is not None:
                states.append((before, h))
            v = (h * C[t].reshape(G, N)[group]).sum(1) + (0 if D is None else D * u[t])
            y[t] = v if z is None else v * z[t] * _sigmoid(z[t])
        hT[s] = h
    return y, hT


def scan_bwd(u, dt, A, B, C, D, z, bias, dy, lengths, h0=None, dhT=None, softplus=True):
    """-> dict of du, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0"""
    rows, E = u.shape
    N, G = A.shape[1], B.shape[1] // A.shape[1]
    group = np.arange(E) // (E // G)
    kept = []
    scan_fwd(u, dt, A, B, C, D, z, bias, lengths, h0, softplus, kept)
    nan = lambda v: np.full_like(v, np.nan)  # noqa: E731
    r = {"du": nan(u), "ddt": nan(u), "dz": nan(u), "dA": np.zeros_like(A), "dB": nan(B), "dC": nan(C), "dD": np.zeros(E), "ddt_bias": np.zeros(E),
         "dh0": np.zeros((len(lengths), E, N))}
    for s, a, b in _spans(lengths):
        g = np.zeros((E, N)) if dhT is None else dhT[s].copy()
        for t in range(b - 1, a - 1, -1):
            before, h = kept[t]
            raw = dt[t] + (0 if bias is None else bias)
            delta = _softplus(raw) if softplus else raw
            Bt, Ct = B[t].reshape(G, N)[group], C[t].reshape(G, N)[group]
            gy = dy[t]
            if z is not None:
                sg = _sigmoid(z[t])
                gy = dy[t] * z[t] * sg
                r["dz"][t] = dy[t] * ((h * Ct).sum(1) + (0 if D is None else D * u[t])) * sg * (1 + z[t] * (1 - sg))
            g = g + gy[:, None] * Ct
            a_t = np.exp(delta[:, None] * A)
            q = g * a_t * before
            gB = (g * Bt).sum(1)
            r["du"][t] = delta * gB + (0 if D is None else gy * D)
            dd = u[t] * gB + (q * A).sum(1)
            r["ddt"][t] = dd * _sigmoid(raw) if softplus else dd
            r["dA"] += q * delta[:, None]
            per = lambda v: np.stack([v[group == k].sum(0) for k in range(G)]).reshape(-1)  # noqa: E731
            r["dB"][t] = per(g * (delta * u[t])[:, None])
            r["dC"][t] = per(h * gy[:, None])
            r["dD"] += gy * u[t]
            r["ddt_bias"] += r["ddt"][t]
            g = g * a_t
        r["dh0"][s] = g
    return r
