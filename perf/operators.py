"""The token-sequence layers as cases to time: the short causal convolution, the norm of heads with the position rotation, and the
selective state space scan, each for training (forward and gradients), for prompts and for single tokens.

Token tensors are (rows, channels) with the sequences packed one behind the other: `seqs` of equal length, or, where `ragged`, of
lengths that the offsets tensor gives (one of a single token and an empty one among them).

  conv  train    forward with SiLU, and dx, dw, dbias              prompt   forward from and to a state of the last inputs
        step     one token for each of `seqs` states
  scan  train    forward, keeping what the gradient needs, and every gradient
        prompt   forward from an initial state, and the final state           step   one token for each of `seqs` states
  rot   train    forward and the gradients of queries, keys and both weights   prompt   forward alone

A gradient's incoming gradient comes from prepare(), as in training it comes from the layers behind.
"""
import math
import random

import torch

own = False

_T = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -----------------------------------------------------------------------------------
def _conv(mode, rows, seqs, D, W, dtype="bf16", ragged=False, silu=True):
    return {"op": "conv", "mode": mode, "rows": rows, "seqs": seqs, "D": D, "W": W, "dtype": dtype, "ragged": ragged, "silu": silu}


def _scan(mode, rows, seqs, D, N, G=1, dtype="bf16", ragged=False, gate=True):
    return {"op": "scan", "mode": mode, "rows": rows, "seqs": seqs, "D": D, "N": N, "G": G, "dtype": dtype, "ragged": ragged, "gate": gate}


def _rot(mode, rows, Hq, Hk, Dh, rot, dtype="bf16", interleaved=False, far=4096):
    return {"op": "rot", "mode": mode, "rows": rows, "Hq": Hq, "Hk": Hk, "Dh": Dh, "rot": rot, "dtype": dtype, "interleaved": interleaved, "far": far}


def listed():
    cases = {
        # one token for each of four streams: the smallest call, all latency
        "conv_step_4": _conv("step", 4, 4, 1024, 4),
        # a training step's convolution: 8 sequences of 2048 tokens
        "conv_train_8x2048": _conv("train", 16384, 8, 4096, 4),
        # prompts of unlike lengths in one batch, fp32, a channel count that is no multiple of a vector
        "conv_prompt_ragged_f32": _conv("prompt", 5003, 13, 1001, 3, "f32", True),
        # one token for each of 64 streams
        "scan_step_64": _scan("step", 64, 64, 4096, 16),
        # prompts of unlike lengths in one batch, from and to the streams' states
        "scan_prompt_ragged": _scan("prompt", 6000, 17, 2048, 16, 1, "bf16", True),
        # one long document
        "scan_prompt_long": _scan("prompt", 32768, 1, 1024, 16),
        # the training step's scan, the largest case
        "scan_train_8x2048": _scan("train", 16384, 8, 2048, 16),
        # a small fp32 model's scan: odd sizes, grouped B and C, half the states, no gate
        "scan_train_odd_f32": _scan("train", 1551, 3, 204, 8, 2, "f32", False, False),
        # one sequence and few channels, so the work is along the tokens: 32 states in four groups
        "scan_train_long": _scan("train", 8193, 1, 512, 32, 4),
        # a few tokens' queries and keys
        "rot_prompt_32": _rot("prompt", 32, 16, 4, 64, 64, far=1000000),
        # a training step's queries and keys
        "rot_train_16384": _rot("train", 16384, 32, 8, 128, 128),
        # the scan's own B and C: groups of 16 states, rotated in part, neighbours paired, fp32
        "rot_train_states_f32": _rot("train", 4099, 8, 8, 16, 8, "f32", True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op, dtype, ragged = rng.choice(["conv", "scan", "scan", "rot"]), rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5
    mode = rng.choice(["train", "train", "prompt", "step"])
    if op == "rot":
        Dh = rng.choice([16, 32, 64, 80, 96, 128, 256])
        return _rot("prompt" if mode == "step" else mode, _log(rng, 1, 32768), rng.randint(1, 32), rng.randint(1, 8), Dh,
                    rng.choice([Dh, Dh, Dh // 2]), dtype, rng.random() < 0.3, rng.choice([4096, 1000000]))
    seqs = _log(rng, 1, 256) if mode == "step" else _log(rng, 1, 32)
    rows = seqs if mode == "step" else seqs * _log(rng, 1, 32768 // seqs)
    if ragged and mode != "step":
        rows = max(seqs, rows + rng.randint(-seqs, seqs))
    D = _log(rng, 64, 4096)
    D = D if rng.random() < 0.25 else max(64, D // 64 * 64)
    if op == "conv":
        return _conv(mode, rows, seqs, D, rng.randint(2, 5), dtype, ragged and mode != "step", rng.random() < 0.8)
    G = rng.choice([1, 1, 1, 2, 4])
    return _scan(mode, rows, seqs, max(G, D // G * G), rng.choice([16, 16, 8, 32, 5]), G, dtype, ragged and mode != "step", rng.random() < 0.7)


def draw(rng):
    """A case of one of the ranges above, its rows cut until it costs no more than the largest listed one of its operator."""
    c = _draw(rng)
    most = max((work(k)["flops"], work(k)["bytes"]) for k in listed() if k["op"] == c["op"])
    while work(c)["flops"] > most[0] or work(c)["bytes"] > most[1]:
        if c["op"] == "rot" or c["ragged"]:
            c["rows"] = max(1, c["rows"] // 2)
        elif c["mode"] == "step":
            c["rows"] = c["seqs"] = max(1, c["seqs"] // 2)
        else:
            c["rows"] = max(1, c["rows"] // c["seqs"] // 2) * c["seqs"]
    return c


def work(c):
    """Each input read once, each output written once; multiplications and additions counted as such, exp and log as one each."""
    b = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rot":
        E = c["rows"] * (c["Hq"] + c["Hk"]) * c["Dh"]
        return {"bytes": (4 if c["mode"] == "train" else 2) * E * b + 4 * c["rows"], "flops": (24 if c["mode"] == "train" else 8) * E}
    E = c["rows"] * c["D"]
    if c["op"] == "conv":
        state = c["seqs"] * (c["W"] - 1) * c["D"] * b
        weights = c["D"] * (c["W"] * b + 4)
        if c["mode"] == "train":
            return {"bytes": 4 * E * b + 2 * weights, "flops": E * (8 * c["W"] + 24)}
        return {"bytes": 2 * E * b + 2 * state + weights, "flops": E * (2 * c["W"] + 5)}
    gate, bc = int(c["gate"]), 2 * c["rows"] * c["G"] * c["N"] * b
    state, weights = 4 * c["seqs"] * c["D"] * c["N"], 4 * c["D"] * (c["N"] + 2)
    if c["mode"] == "train":
        return {"bytes": 2 * (3 + gate) * E * b + 2 * bc + 2 * weights, "flops": E * c["N"] * 26 + 30 * E}
    return {"bytes": (3 + gate) * E * b + bc + 2 * state + weights, "flops": E * c["N"] * 7 + 12 * E}


# ---- inputs --------------------------------------------------------------------------------------
def _lengths(rows, seqs, seed):
    """seqs lengths that add up to rows: one empty and one of a single token where there are enough."""
    r = random.Random(seed * 7919 + rows)
    if seqs < 4 or rows < seqs:
        cuts = sorted(r.randint(0, rows) for _ in range(seqs - 1))
        return [b - a for a, b in zip([0] + cuts, cuts + [rows])]
    share = [r.uniform(0.1, 1) ** 2 for _ in range(seqs - 2)]
    left = rows - 1
    got = [int(left * s / sum(share)) for s in share]
    got[0] += left - sum(got)
    got += [0, 1]
    r.shuffle(got)
    return got


def _offsets(c, seed):
    if not c.get("ragged"):
        return None
    at = [0]
    for n in _lengths(c["rows"], c["seqs"], seed):
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = _T[c["dtype"]]

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=g, device="cuda") * (hi - lo) + lo

    rows, s = c["rows"], {"case": dict(c)}
    if c["op"] == "rot":
        Dh = c["Dh"]
        s.update(q=normal(rows, c["Hq"] * Dh), k=normal(rows, c["Hk"] * Dh), wq=uniform(0.5, 1.5, Dh), wk=uniform(0.5, 1.5, Dh),
                 positions=torch.randint(0, c["far"], (rows,), generator=g, device="cuda", dtype=torch.int32),
                 inv_freq=(10000.0 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64) * 2 / c["rot"])).float().cuda())
        s.update(yq=torch.empty_like(s["q"]), yk=torch.empty_like(s["k"]))
        if c["mode"] == "train":
            s.update(dyq=normal(rows, c["Hq"] * Dh), dyk=normal(rows, c["Hk"] * Dh), dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]),
                     dwq=torch.empty_like(s["wq"]), dwk=torch.empty_like(s["wk"]))
            if own:
                import paper_1801_04380_amd as sn
                s["scratch"] = torch.empty(sn.sn_headnorm_rot_scratch_bytes(rows, c["Hq"], c["Hk"], Dh), dtype=torch.uint8, device="cuda")
        return s

    D, seqs = c["D"], c["seqs"]
    s["offsets"] = _offsets(c, seed)
    if c["op"] == "conv":
        W = c["W"]
        s.update(x=normal(rows, D), w=normal(D, W, scale=W ** -0.5), bias=normal(D, scale=0.1, dtype=torch.float32))
        s["y"] = torch.empty_like(s["x"])
        if c["mode"] != "train":
            s["state"] = normal(seqs, W - 1, D)
            s["state_out"] = torch.empty_like(s["state"])
        if c["mode"] == "step":
            s["slots"] = torch.randperm(seqs, generator=g, device="cuda").to(torch.int32)
        if c["mode"] == "train":
            s.update(dy=normal(rows, D), dx=torch.empty_like(s["x"]), dw=torch.empty(D, W, device="cuda"), dbias=torch.empty(D, device="cuda"))
            if own:
                import paper_1801_04380_amd as sn
                s["scratch"] = torch.empty(sn.sn_causal_conv1d_scratch_bytes(rows, D, W), dtype=torch.uint8, device="cuda")
        return s

    N, G = c["N"], c["G"]
    step = torch.exp(uniform(math.log(1e-3), math.log(1e-1), D))
    s.update(u=normal(rows, D, scale=0.5), dt=normal(rows, D, scale=0.5), B=normal(rows, G * N), C=normal(rows, G * N),
             A=-(torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * uniform(0.5, 1.5, D, 1)), D=uniform(0.5, 1.5, D),
             dt_bias=step + torch.log(-torch.expm1(-step)), z=normal(rows, D) if c["gate"] else None)
    s["y"] = torch.empty_like(s["u"])
    if c["mode"] != "train":
        s["h0"] = normal(seqs, D, N, scale=0.1, dtype=torch.float32)
        s["hT"] = torch.empty_like(s["h0"])
    if c["mode"] == "step":
        s["slots"] = torch.randperm(seqs, generator=g, device="cuda").to(torch.int32)
    if c["mode"] == "train":
        s.update(dy=normal(rows, D), du=torch.empty_like(s["u"]), ddt=torch.empty_like(s["u"]), dA=torch.empty_like(s["A"]),
                 dB=torch.empty_like(s["B"]), dC=torch.empty_like(s["C"]), dD=torch.empty_like(s["D"]),
                 dz=torch.empty_like(s["u"]) if c["gate"] else None, ddt_bias=torch.empty_like(s["D"]))
    if own and c["mode"] != "step":
        import paper_1801_04380_amd as sn
        shape = sn.scan_shape(rows, D, N, G, seqs, sn.SN_BF16 if c["dtype"] == "bf16" else sn.SN_F32, c["ragged"])
        need = sn.sn_scan_workspace_query(shape, sn.SN_SCAN_FWD)[1]
        if c["mode"] == "train":
            s["states"] = torch.empty(sn.sn_scan_states_bytes(shape), dtype=torch.uint8, device="cuda")
            need = max(need, sn.sn_scan_workspace_query(shape, sn.SN_SCAN_BWD)[1])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


# ---- the framework's calls -----------------------------------------------------------------------
def _own(s):
    import paper_1801_04380_amd as sn
    c = s["case"]
    if c["op"] == "rot":
        kw = {"head_dim": c["Dh"], "eps": 1e-6, "interleaved": c["interleaved"]}
        sn.sn_headnorm_rot_fwd(s["q"], s["k"], s["wq"], s["wk"], s["positions"], s["inv_freq"], s["yq"], s["yk"], **kw)
        if c["mode"] != "train":
            return s["yq"], s["yk"]
        sn.sn_headnorm_rot_bwd(s["q"], s["k"], s["wq"], s["wk"], s["positions"], s["inv_freq"], s["dyq"], s["dyk"], s["dq"], s["dk"],
                               s["dwq"], s["dwk"], s["scratch"], **kw)
        return s["yq"], s["yk"], s["dq"], s["dk"], s["dwq"], s["dwk"]
    if c["op"] == "conv":
        if c["mode"] == "step":
            sn.sn_causal_conv1d_step(s["x"], s["w"], s["bias"], s["y"], s["state"], state_out=s["state_out"], slots=s["slots"], silu=c["silu"])
            return s["y"], s["state_out"]
        if c["mode"] == "prompt":
            sn.sn_causal_conv1d_fwd(s["x"], s["w"], s["bias"], s["y"], offsets=s["offsets"], seqs=c["seqs"], state_in=s["state"],
                                    state_out=s["state_out"], silu=c["silu"])
            return s["y"], s["state_out"]
        sn.sn_causal_conv1d_fwd(s["x"], s["w"], s["bias"], s["y"], offsets=s["offsets"], seqs=c["seqs"], silu=c["silu"])
        sn.sn_causal_conv1d_bwd(s["x"], s["w"], s["bias"], s["dy"], s["dx"], s["dw"], s["dbias"], s["scratch"], offsets=s["offsets"],
                                seqs=c["seqs"], silu=c["silu"])
        return s["y"], s["dx"], s["dw"], s["dbias"]
    data = [s[k] for k in ("u", "dt", "A", "B", "C", "D", "z", "dt_bias")]
    if c["mode"] == "step":
        sn.sn_scan_step(*data, s["y"], s["h0"], state_out=s["hT"], slots=s["slots"])
        return s["y"], s["hT"]
    if c["mode"] == "prompt":
        sn.sn_scan_fwd(*data, s["y"], offsets=s["offsets"], seqs=c["seqs"], h0=s["h0"], hT=s["hT"], workspace=s["workspace"])
        return s["y"], s["hT"]
    sn.sn_scan_fwd(*data, s["y"], offsets=s["offsets"], seqs=c["seqs"], states=s["states"], workspace=s["workspace"])
    sn.sn_scan_bwd(*data, s["dy"], s["du"], s["ddt"], s["dA"], s["dB"], s["dC"], s["dD"], s["dz"], s["ddt_bias"], s["workspace"],
                   offsets=s["offsets"], seqs=c["seqs"], states=s["states"])
    return tuple(s[k] for k in ("y", "du", "ddt", "dA", "dB", "dC", "dD", "ddt_bias") + (("dz",) if c["gate"] else ()))


# ---- the plain forms -----------------------------------------------------------------------------
def _places(s):
    """The sequence of every row and the offsets."""
    c = s["case"]
    off = s["offsets"]
    if off is None:
        off = torch.arange(c["seqs"] + 1, device="cuda", dtype=torch.int32) * (c["rows"] // c["seqs"])
    return torch.searchsorted(off, torch.arange(c["rows"], device="cuda", dtype=torch.int32), right=True) - 1, off.long()


def _rms_rotate(x, w, cos, sin, heads, c):
    """The normalised heads, rotated, in 32 bits; and 1 / rms."""
    x = x.float().view(x.shape[0], heads, c["Dh"])
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    return _rotate(x * r * w, cos, sin, c), r


def _rotate(n, cos, sin, c):
    rot, y = c["rot"], n.clone()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., one] = n[..., one] * cos - n[..., two] * sin
    y[..., two] = n[..., two] * cos + n[..., one] * sin
    return y


def _rms_rotate_back(x, r, w, dy, cos, sin, heads, c):
    x, g = x.float().view(x.shape[0], heads, c["Dh"]), _rotate(dy.float().view(x.shape[0], heads, c["Dh"]), cos, -sin, c)
    gw = g * w
    dx = r * (gw - x * r * r * (gw * x).mean(-1, keepdim=True))
    return dx.flatten(1), (g * x * r).sum((0, 1))


def _plain_rot(s):
    c, t = s["case"], s["q"].dtype
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    yq, rq = _rms_rotate(s["q"], s["wq"], cos, sin, c["Hq"], c)
    yk, rk = _rms_rotate(s["k"], s["wk"], cos, sin, c["Hk"], c)
    yq, yk = yq.flatten(1).to(t), yk.flatten(1).to(t)
    if c["mode"] != "train":
        return yq, yk
    dq, dwq = _rms_rotate_back(s["q"], rq, s["wq"], s["dyq"], cos, sin, c["Hq"], c)
    dk, dwk = _rms_rotate_back(s["k"], rk, s["wk"], s["dyk"], cos, sin, c["Hk"], c)
    return yq, yk, dq.to(t), dk.to(t), dwq, dwk


def _plain_conv_step(s):
    c, t = s["case"], s["x"].dtype
    slots = s["slots"].long()
    taps = torch.cat((s["state"][slots], s["x"][:, None]), 1)
    p = (taps.float() * s["w"].float().t()).sum(1) + s["bias"]
    new = torch.empty_like(s["state"])
    new[slots] = taps[:, 1:]
    return (p * torch.sigmoid(p) if c["silu"] else p).to(t), new


def _plain_conv(s):
    c, t, W = s["case"], s["x"].dtype, s["case"]["W"]
    if c["mode"] == "step":
        return _plain_conv_step(s)
    seq, off = _places(s)
    row = torch.arange(c["rows"], device="cuda")
    back = torch.arange(W - 1, -1, -1, device="cuda")
    src = row[:, None] - back                                    # (rows, W): the row under each tap
    inside = src >= off[seq][:, None]
    taps = s["x"].float()[src.clamp_min(0)] * inside[..., None]  # (rows, W, D)
    if c["mode"] == "prompt":
        old = s["state"].float()[seq[:, None], (W - 1 + src - off[seq][:, None]).clamp(0, W - 2)]
        taps = torch.where(inside[..., None], taps, old)
    w = s["w"].float()
    p = (taps * w.t()).sum(1) + s["bias"]
    sig = torch.sigmoid(p)
    y = (p * sig if c["silu"] else p).to(t)
    if c["mode"] == "prompt":
        end = off[1:, None] - torch.arange(W - 1, 0, -1, device="cuda")
        has = end >= off[:-1, None]
        old = torch.gather(s["state"], 1, (W - 1 + end - off[:-1, None]).clamp(0, W - 2)[..., None].expand(-1, -1, c["D"]))
        return y, torch.where(has[..., None], s["x"][end.clamp_min(0)], old)
    dp = s["dy"].float()
    if c["silu"]:
        dp = dp * (sig + p * sig * (1 - sig))
    dst = row[:, None] + back
    same = (dst < off[seq + 1][:, None])[..., None]
    dx = (dp[dst.clamp_max(c["rows"] - 1)] * same * w.t()).sum(1)
    return y, dx.to(t), (taps * dp[:, None]).sum(0).t().contiguous(), dp.sum(0)


def _recur(a, b, length):
    """h[t] = a[t] h[t-1] + b[t] along the rows, by doubling."""
    k = 1
    while k < length:
        b = torch.cat((b[:k], torch.addcmul(b[k:], a[k:], b[:-k])))
        a = torch.cat((a[:k], a[k:] * a[:-k]))
        k *= 2
    return b


def _plain_scan_step(s):
    c, t, D, N = s["case"], s["u"].dtype, s["case"]["D"], s["case"]["N"]
    slots = s["slots"].long()
    u, each = s["u"].float(), D // c["G"]
    delta = torch.logaddexp(s["dt"].float() + s["dt_bias"], torch.zeros((), device="cuda"))
    B, C = (s[k].float().view(-1, c["G"], N).repeat_interleave(each, 1) for k in ("B", "C"))
    h = torch.exp(delta[..., None] * s["A"]) * s["h0"][slots] + (delta * u)[..., None] * B
    y = (h * C).sum(-1) + s["D"] * u
    if c["gate"]:
        z = s["z"].float()
        y = y * z * torch.sigmoid(z)
    new = torch.empty_like(s["h0"])
    new[slots] = h
    return y.to(t), new


def _plain_scan(s):
    c, t, D, N, G, T = s["case"], s["u"].dtype, s["case"]["D"], s["case"]["N"], s["case"]["G"], s["case"]["rows"]
    if c["mode"] == "step":
        return _plain_scan_step(s)
    seq, off = _places(s)
    first = torch.ones(T, dtype=torch.bool, device="cuda")
    first[1:] = seq[1:] != seq[:-1]
    length = T if c["ragged"] else T // c["seqs"]
    u, each = s["u"].float(), D // G
    raw = s["dt"].float() + s["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros((), device="cuda"))
    B, C = (s[k].float().view(T, G, 1, N) for k in ("B", "C"))
    a = torch.exp(delta[..., None] * s["A"])
    b = ((delta * u).view(T, G, each, 1) * B).view(T, D, N)
    if c["mode"] == "prompt":
        b = torch.where(first[:, None, None], b + a * s["h0"][seq], b)
    stay = torch.where(first[:, None, None], torch.zeros((), device="cuda"), a)
    h = _recur(stay, b, length)
    del b
    y = (h.view(T, G, each, N) * C).sum(-1).view(T, D) + s["D"] * u
    gate = torch.ones((), device="cuda")
    if c["gate"]:
        z = s["z"].float()
        sig = torch.sigmoid(z)
        gate = z * sig
    out = (y * gate).to(t)
    if c["mode"] == "prompt":
        some = (off[1:] > off[:-1])[:, None, None]
        return out, torch.where(some, h[(off[1:] - 1).clamp_min(0)], s["h0"])
    dy = s["dy"].float()
    gy = dy * gate
    # the gradient of h runs the other way: g[t] = gy[t] C[t] + a[t+1] g[t+1]
    after = torch.cat((stay[1:], torch.zeros(1, D, N, device="cuda")))
    g = _recur(after.flip(0), (gy.view(T, G, each, 1) * C).view(T, D, N).flip(0), length).flip(0)
    del after
    before = torch.cat((torch.zeros(1, D, N, device="cuda"), h[:-1])) * stay   # a[t] h[t-1]
    dC = (gy.view(T, G, each, 1) * h.view(T, G, each, N)).sum(2).reshape(T, G * N)
    del h, stay, a
    gB = (g.view(T, G, each, N) * B).sum(-1).view(T, D)
    dB = (g.view(T, G, each, N) * (delta * u).view(T, G, each, 1)).sum(2).reshape(T, G * N)
    q = g * before
    del g, before
    ddelta = gB * u + (q * s["A"]).sum(-1)
    ddt = ddelta * torch.sigmoid(raw)
    found = [out, (gB * delta + gy * s["D"]).to(t), ddt.to(t), (q * delta[..., None]).sum(0), dB.to(t), dC.to(t), (gy * u).sum(0), ddt.sum(0)]
    if c["gate"]:
        found.append((dy * y * (sig + z * sig * (1 - sig))).to(t))
    return tuple(found)


def run(state):
    if own:
        return _own(state)
    return {"rot": _plain_rot, "conv": _plain_conv, "scan": _plain_scan}[state["case"]["op"]](state)


# ---- the definitions in 64 bits, token after token -----------------------------------------------
def _padded(x, lengths):
    """(rows, ...) -> (seqs, longest, ...) in 64 bits, zero behind each sequence's end."""
    x = x.double()
    y = torch.zeros((len(lengths), max(1, max(lengths))) + tuple(x.shape[1:]), dtype=torch.float64, device=x.device)
    at = 0
    for i, n in enumerate(lengths):
        y[i, :n] = x[at:at + n]
        at += n
    return y


def _packed(x, lengths):
    return torch.cat([x[i, :n] for i, n in enumerate(lengths)])


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rot":
        return _exact_rot(s, c)
    if c["mode"] == "step":
        lengths = [1] * c["seqs"]
    elif c["ragged"]:
        lengths = _lengths(c["rows"], c["seqs"], seed)
    else:
        lengths = [c["rows"] // c["seqs"]] * c["seqs"]
    if c["op"] == "scan" and 8.0 * len(lengths) * max(lengths) * c["D"] * c["N"] * 3 > 100e9:
        return None
    order = s["slots"].long() if c["mode"] == "step" else torch.arange(c["seqs"], device="cuda")
    return (_exact_conv if c["op"] == "conv" else _exact_scan)(s, c, lengths, order)


def _exact_rot(s, c):
    """By complex numbers: a pair is a number, the rotation a product with exp(i * angle)."""
    half = c["rot"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]

    def rotated(v, by):
        if c["interleaved"]:
            head = torch.view_as_real(torch.complex(v[..., 0:c["rot"]:2].contiguous(), v[..., 1:c["rot"]:2].contiguous()) * by).flatten(-2)
        else:
            p = torch.complex(v[..., :half].contiguous(), v[..., half:c["rot"]].contiguous()) * by
            head = torch.cat((p.real, p.imag), -1)
        return torch.cat((head, v[..., c["rot"]:]), -1)

    def one(x, w, heads, dy):
        x, w = x.double().view(c["rows"], heads, c["Dh"]), w.double()
        rms = (x.pow(2).sum(-1, keepdim=True) / c["Dh"] + 1e-6).sqrt()
        y = rotated(x / rms * w, turn).flatten(1)
        if dy is None:
            return y, None, None
        g = rotated(dy.double().view(c["rows"], heads, c["Dh"]), turn.conj())
        xhat = x / rms
        dx = (g * w - xhat * (g * w * xhat).sum(-1, keepdim=True) / c["Dh"]) / rms
        return y, dx.flatten(1), (g * xhat).sum((0, 1))

    yq, dq, dwq = one(s["q"], s["wq"], c["Hq"], s.get("dyq"))
    yk, dk, dwk = one(s["k"], s["wk"], c["Hk"], s.get("dyk"))
    return (yq, yk) if c["mode"] != "train" else (yq, yk, dq, dk, dwq, dwk)


def _exact_conv(s, c, lengths, order):
    W, D = c["W"], c["D"]
    x = _padded(s["x"], lengths)
    old = s["state"].double()[order] if c["mode"] != "train" else torch.zeros(len(lengths), W - 1, D, dtype=torch.float64, device="cuda")
    line = torch.cat((old, x), 1)                       # (seqs, W - 1 + longest, D)
    L, w = x.shape[1], s["w"].double()
    p = s["bias"].double() + sum(line[:, j:j + L] * w[:, j] for j in range(W))
    y = p / (1 + torch.exp(-p)) if c["silu"] else p
    if c["mode"] != "train":
        new = torch.empty_like(old)
        for i, n in enumerate(lengths):
            new[order[i]] = line[i, n:n + W - 1]
        return _packed(y, lengths), new
    dp = _padded(s["dy"], lengths)
    if c["silu"]:
        sig = 1 / (1 + torch.exp(-p))
        dp = dp * sig * (1 + p * (1 - sig))
    dline = torch.zeros_like(line)
    for j in range(W):
        dline[:, j:j + L] += dp * w[:, j]
    dw = torch.stack([(dp * line[:, j:j + L]).sum((0, 1)) for j in range(W)], 1)
    return _packed(y, lengths), _packed(dline[:, W - 1:], lengths), dw, dp.sum((0, 1))


def _exact_scan(s, c, lengths, order):
    D, N, G = c["D"], c["N"], c["G"]
    u, raw = _padded(s["u"], lengths), _padded(s["dt"], lengths) + s["dt_bias"].double()
    S, L, each = u.shape[0], u.shape[1], D // G
    alive = (torch.arange(L, device="cuda") < torch.tensor(lengths, device="cuda")[:, None])[..., None]
    delta = torch.where(raw > 30, raw, torch.log1p(torch.exp(raw.clamp(max=30)))) * alive   # 0 behind the end: h stays
    B, C = (_padded(s[k], lengths).view(S, L, G, 1, N) for k in ("B", "C"))
    A = s["A"].double()
    h = s["h0"].double()[order] if c["mode"] != "train" else torch.zeros(S, D, N, dtype=torch.float64, device="cuda")
    y, kept = torch.empty_like(u), []
    for i in range(L):
        if c["mode"] == "train":
            kept.append(h)
        d = delta[:, i, :, None]
        h = torch.exp(d * A) * h + ((delta[:, i] * u[:, i]).view(S, G, each, 1) * B[:, i]).view(S, D, N)
        y[:, i] = (h.view(S, G, each, N) * C[:, i]).sum(-1).view(S, D)
    y += s["D"].double() * u
    out = y
    if c["gate"]:
        z = _padded(s["z"], lengths)
        sig = 1 / (1 + torch.exp(-z))
        out = y * z * sig
    if c["mode"] != "train":
        new = torch.empty_like(h)
        new[order] = h
        return _packed(out, lengths), new
    dy = _padded(s["dy"], lengths)
    gy = dy * z * sig if c["gate"] else dy
    g, dA = torch.zeros_like(h), torch.zeros_like(A)
    du, dd, dB, dC = s["D"].double() * gy, torch.empty_like(u), torch.empty_like(B[:, :, :, 0]), torch.empty_like(B[:, :, :, 0])
    for i in range(L - 1, -1, -1):
        d, past = delta[:, i, :, None], kept.pop()
        decayed = torch.exp(d * A) * past
        now = decayed + ((delta[:, i] * u[:, i]).view(S, G, each, 1) * B[:, i]).view(S, D, N)
        g = g + (gy[:, i].view(S, G, each, 1) * C[:, i]).view(S, D, N)
        dC[:, i] = (now * gy[:, i, :, None]).view(S, G, each, N).sum(2)
        dB[:, i] = (g * (delta[:, i] * u[:, i])[..., None]).view(S, G, each, N).sum(2)
        gB = (g.view(S, G, each, N) * B[:, i]).sum(-1).view(S, D)
        du[:, i] += gB * delta[:, i]
        dd[:, i] = gB * u[:, i] + (g * decayed * A).sum(-1)
        dA += (g * decayed * d).sum(0)
        g = g * torch.exp(d * A)
    ddt = dd / (1 + torch.exp(-raw)) * alive
    found = [_packed(out, lengths), _packed(du, lengths), _packed(ddt, lengths), dA, _packed(dB, lengths).flatten(1), _packed(dC, lengths).flatten(1),
             (gy * u).sum((0, 1)), ddt.sum((0, 1))]
    if c["gate"]:
        found.append(_packed(dy * y * sig * (1 + z * (1 - sig)), lengths))
    return tuple(found)
