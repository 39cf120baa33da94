"""Python names for the C ABI of include/sn_seq.h (argument marshalling only): layers along token sequences.

Token tensors are torch CUDA (ROCm) tensors of shape (rows, channels), channels contiguous, rows any stride apart; each
call runs on torch's current stream, and its tensors have to live on the current device.  Nothing here computes anything.
"""
import ctypes

import torch

from . import _lib
from .api import SN_BF16, SN_F32, _check, _dtype_code, _stream

__all__ = [
    "sn_causal_conv1d_fwd", "sn_causal_conv1d_scratch_bytes", "sn_causal_conv1d_bwd", "sn_causal_conv1d_step",
    "sn_headnorm_rot_fwd", "sn_headnorm_rot_scratch_bytes", "sn_headnorm_rot_bwd",
    "SN_SCAN_FWD", "SN_SCAN_BWD", "scan_shape", "sn_scan_workspace_query", "sn_scan_states_bytes", "sn_scan_fwd",
    "sn_scan_bwd", "sn_scan_step",
]

_vp, _sz, _i, _i32, _i64, _f = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
SN_SCAN_FWD, SN_SCAN_BWD = 0, 1


class Conv1dShape(ctypes.Structure):
    """Mirror of sn_conv1d_shape."""
    _fields_ = [("rows", _i64)] + [(n, _i32) for n in ("seqs", "channels", "width", "silu", "dtype")] + [
        (n, _i64) for n in ("ld_x", "ld_y", "ld_dx")]


class HeadnormShape(ctypes.Structure):
    """Mirror of sn_headnorm_shape."""
    _fields_ = [("rows", _i64)] + [(n, _i32) for n in ("q_heads", "k_heads", "head_dim", "rot_dim", "interleaved", "dtype")] + [
        ("eps", _f)] + [(n, _i64) for n in ("ld_q", "ld_k", "ld_yq", "ld_yk", "ld_dq", "ld_dk")]


class ScanShape(ctypes.Structure):
    """Mirror of sn_scan_shape."""
    _fields_ = [("rows", _i64)] + [(n, _i32) for n in ("seqs", "channels", "states", "groups", "dtype", "softplus", "ragged")] + [
        (n, _i64) for n in ("ld_u", "ld_dt", "ld_b", "ld_c", "ld_z", "ld_y", "ld_du", "ld_ddt", "ld_db", "ld_dc", "ld_dz")]


_c1, _hn, _sc = ctypes.POINTER(Conv1dShape), ctypes.POINTER(HeadnormShape), ctypes.POINTER(ScanShape)

# name -> (restype, argtypes); every symbol include/sn_seq.h declares
SIGNATURES = {
    "sn_causal_conv1d_fwd": (_i, [_vp] * 4 + [_c1] + [_vp] * 4),
    "sn_causal_conv1d_scratch_bytes": (_sz, [_i64, _i32, _i32]),
    "sn_causal_conv1d_bwd": (_i, [_vp] * 7 + [_c1] + [_vp] * 5 + [_sz, _vp]),
    "sn_causal_conv1d_step": (_i, [_vp] * 7 + [_i32, _c1, _vp]),
    "sn_headnorm_rot_fwd": (_i, [_vp] * 8 + [_hn, _vp]),
    "sn_headnorm_rot_scratch_bytes": (_sz, [_i64, _i32, _i32, _i32]),
    "sn_headnorm_rot_bwd": (_i, [_vp] * 12 + [_hn, _vp, _sz, _vp]),
    "sn_scan_workspace_query": (_i, [_sc, _i, ctypes.POINTER(_sz), ctypes.POINTER(_sz)]),
    "sn_scan_states_bytes": (_sz, [_sc]),
    "sn_scan_fwd": (_i, [_vp] * 9 + [_sc] + [_vp] * 5 + [_sz, _vp]),
    "sn_scan_bwd": (_i, [_vp] * 17 + [_sc] + [_vp] * 6 + [_sz, _vp]),
    "sn_scan_step": (_i, [_vp] * 12 + [_i32, _sc, _vp]),
}

_fns = {}


def _fn(name):
    f = _fns.get(name)
    if f is None:
        f = getattr(_lib.load(), name)
        f.restype, f.argtypes = SIGNATURES[name]
        _fns[name] = f
    return f


def _call(name, *args):
    _check(name, _fn(name)(*args))


def _here(t, what):
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError("%s: expected a tensor on the current device" % what)


def _rows(t, rows, width, dtype, what):
    """-> (pointer, row stride) of a (rows, width) token tensor."""
    _here(t, what)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != width or t.dtype != dtype:
        raise ValueError("%s: expected a (%d, %d) tensor of %s, got %s of %s" % (what, rows, width, dtype, tuple(t.shape), t.dtype))
    if width > 1 and t.stride(1) != 1:
        raise ValueError("%s: the channels of a row have to be contiguous" % what)
    return t.data_ptr(), t.stride(0)


def _dense(t, shape, dtype, what):
    """-> pointer of a contiguous tensor of that shape, None for None."""
    if t is None:
        return None
    _here(t, what)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous %s tensor of %s, got %s of %s" % (what, tuple(shape), dtype, tuple(t.shape), t.dtype))
    return t.data_ptr()


def _bytes(t, what):
    if t is None:
        return None, 0
    _here(t, what)
    if not t.is_contiguous():
        raise ValueError("%s: expected a contiguous tensor" % what)
    return t.data_ptr(), t.numel() * t.element_size()


def _offsets(offsets, seqs):
    return _dense(offsets, (seqs + 1,), torch.int32, "offsets")


def _slots(slots, rows):
    return _dense(slots, (rows,), torch.int32, "slots")


# ---- short causal convolution ----
def _conv1d_shape(x, w, y, what, seqs, silu, dx=None):
    rows, channels = x.shape
    width = w.shape[1]
    xp, ldx = _rows(x, rows, channels, x.dtype, "x")
    yp, ldy = _rows(y, rows, channels, x.dtype, what)
    dxp, lddx = _rows(dx, rows, channels, x.dtype, "dx") if dx is not None else (None, 0)
    wp = _dense(w, (channels, width), x.dtype, "w")
    return xp, wp, yp, dxp, Conv1dShape(rows, seqs, channels, width, int(bool(silu)), _dtype_code(x), ldx, ldy, lddx)


def sn_causal_conv1d_fwd(x, w, bias, y, offsets=None, seqs=1, state_in=None, state_out=None, silu=True):
    xp, wp, yp, _, s = _conv1d_shape(x, w, y, "y", seqs, silu)
    state = (seqs, s.width - 1, s.channels)
    _call("sn_causal_conv1d_fwd", xp, wp, _dense(bias, (s.channels,), torch.float32, "bias"), yp, ctypes.byref(s), _offsets(offsets, seqs),
          _dense(state_in, state, x.dtype, "state_in"), _dense(state_out, state, x.dtype, "state_out"), _stream())


def sn_causal_conv1d_scratch_bytes(rows, channels, width):
    return int(_fn("sn_causal_conv1d_scratch_bytes")(rows, channels, width))


def sn_causal_conv1d_bwd(x, w, bias, dy, dx, dw, dbias, scratch, offsets=None, seqs=1, state_in=None, dstate_out=None, dstate_in=None, silu=True):
    xp, wp, gp, dxp, s = _conv1d_shape(x, w, dy, "dy", seqs, silu, dx)
    state, vec = (seqs, s.width - 1, s.channels), (s.channels,)
    sp, sb = _bytes(scratch, "scratch")
    _call("sn_causal_conv1d_bwd", xp, wp, _dense(bias, vec, torch.float32, "bias"), gp, dxp, _dense(dw, (s.channels, s.width), torch.float32, "dw"),
          _dense(dbias, vec, torch.float32, "dbias"), ctypes.byref(s), _offsets(offsets, seqs), _dense(state_in, state, x.dtype, "state_in"),
          _dense(dstate_out, state, x.dtype, "dstate_out"), _dense(dstate_in, state, x.dtype, "dstate_in"), sp, sb, _stream())


def sn_causal_conv1d_step(x, w, bias, y, state, state_out=None, slots=None, silu=True):
    """One token for each row of x; state: (num_slots, width - 1, channels), updated in place unless state_out is given."""
    xp, wp, yp, _, s = _conv1d_shape(x, w, y, "y", 1, silu)
    shape = (state.shape[0], s.width - 1, s.channels)
    sp = _dense(state, shape, x.dtype, "state")
    _call("sn_causal_conv1d_step", xp, wp, _dense(bias, (s.channels,), torch.float32, "bias"), yp, sp,
          sp if state_out is None else _dense(state_out, shape, x.dtype, "state_out"), _slots(slots, s.rows), shape[0], ctypes.byref(s), _stream())


# ---- norm of heads and position rotation ----
def _headnorm_shape(q, k, yq, yk, inv_freq, head_dim, eps, interleaved, dq=None, dk=None):
    rows, nq = q.shape
    nk = k.shape[1] if k is not None else 0
    if head_dim < 1 or nq % head_dim or nk % head_dim:
        raise ValueError("the rows of q and k have to hold whole heads of head_dim = %d" % head_dim)
    none = (None, 0)
    ptrs = [_rows(t, rows, n, q.dtype, what) if t is not None else none
            for t, n, what in ((q, nq, "q"), (k, nk, "k"), (yq, nq, "yq"), (yk, nk, "yk"), (dq, nq, "dq"), (dk, nk, "dk"))]
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    s = HeadnormShape(rows, nq // head_dim, nk // head_dim, head_dim, rot, int(bool(interleaved)), _dtype_code(q), eps, *(p[1] for p in ptrs))
    return [p[0] for p in ptrs], s


def _headnorm_args(wq, wk, positions, inv_freq, s):
    return (_dense(wq, (s.head_dim,), torch.float32, "wq"), _dense(wk, (s.head_dim,), torch.float32, "wk"),
            _dense(positions, (s.rows,), torch.int32, "positions"), _dense(inv_freq, (s.rot_dim // 2,), torch.float32, "inv_freq"))


def sn_headnorm_rot_fwd(q, k, wq, wk, positions, inv_freq, yq, yk, head_dim, eps=1e-6, interleaved=False):
    """q, k: (rows, heads * head_dim); k and yk may be None.  inv_freq has rot_dim / 2 elements, or is None for no rotation."""
    (qp, kp, yqp, ykp, _, _), s = _headnorm_shape(q, k, yq, yk, inv_freq, head_dim, eps, interleaved)
    _call("sn_headnorm_rot_fwd", qp, kp, *_headnorm_args(wq, wk, positions, inv_freq, s), yqp, ykp, ctypes.byref(s), _stream())


def sn_headnorm_rot_scratch_bytes(rows, q_heads, k_heads, head_dim):
    return int(_fn("sn_headnorm_rot_scratch_bytes")(rows, q_heads, k_heads, head_dim))


def sn_headnorm_rot_bwd(q, k, wq, wk, positions, inv_freq, dyq, dyk, dq, dk, dwq, dwk, scratch, head_dim, eps=1e-6, interleaved=False):
    (qp, kp, gqp, gkp, dqp, dkp), s = _headnorm_shape(q, k, dyq, dyk, inv_freq, head_dim, eps, interleaved, dq, dk)
    vec = (head_dim,)
    sp, sb = _bytes(scratch, "scratch")
    _call("sn_headnorm_rot_bwd", qp, kp, *_headnorm_args(wq, wk, positions, inv_freq, s), gqp, gkp, dqp, dkp,
          _dense(dwq, vec, torch.float32, "dwq"), _dense(dwk, vec, torch.float32, "dwk"), ctypes.byref(s), sp, sb, _stream())


# ---- selective state space scan ----
def scan_shape(rows, channels, states, groups=1, seqs=1, dtype=SN_BF16, ragged=False, softplus=True):
    """The sizes that the queries take; the calls below make theirs from their tensors."""
    return ScanShape(rows, seqs, channels, states, groups, dtype, int(bool(softplus)), int(bool(ragged)))


def sn_scan_workspace_query(shape, direction):
    """-> (min_bytes, preferred_bytes)."""
    mn, pf = ctypes.c_size_t(), ctypes.c_size_t()
    _call("sn_scan_workspace_query", ctypes.byref(shape), direction, ctypes.byref(mn), ctypes.byref(pf))
    return mn.value, pf.value


def sn_scan_states_bytes(shape):
    return int(_fn("sn_scan_states_bytes")(ctypes.byref(shape)))


def _scan_inputs(u, dt, A, B, C, D, z, dt_bias, y, what, seqs, softplus, ragged):
    rows, channels = u.shape
    states = A.shape[1]
    if states < 1 or B.dim() != 2 or B.shape[1] % states:
        raise ValueError("the rows of B and C have to hold whole groups of states = %d" % states)
    t, vec, gn = u.dtype, (channels,), B.shape[1]
    ptrs = [_rows(v, rows, n, t, name) for v, n, name in ((u, channels, "u"), (dt, channels, "dt"), (B, gn, "B"), (C, gn, "C"))]
    ptrs.append(_rows(z, rows, channels, t, "z") if z is not None else (None, 0))
    ptrs.append(_rows(y, rows, channels, t, what))
    s = ScanShape(rows, seqs, channels, states, gn // states, _dtype_code(u), int(bool(softplus)), int(ragged), *(p[1] for p in ptrs))
    up, dtp, bp, cp, zp, yp = (p[0] for p in ptrs)
    return s, (up, dtp, _dense(A, (channels, states), torch.float32, "A"), bp, cp, _dense(D, vec, torch.float32, "D"), zp,
               _dense(dt_bias, vec, torch.float32, "dt_bias"), yp)


def _states(states, s):
    p, n = _bytes(states, "states")
    if states is not None and n < sn_scan_states_bytes(s):
        raise ValueError("states: %d bytes, needs %d" % (n, sn_scan_states_bytes(s)))
    return p


def sn_scan_fwd(u, dt, A, B, C, D, z, dt_bias, y, offsets=None, seqs=1, h0=None, hT=None, states=None, workspace=None, softplus=True):
    """u, dt, z, y: (rows, channels); A: (channels, states); B, C: (rows, groups * states); D, z, dt_bias may be None."""
    s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, y, "y", seqs, softplus, offsets is not None)
    h = (seqs, s.channels, s.states)
    wp, wb = _bytes(workspace, "workspace")
    _call("sn_scan_fwd", *args, ctypes.byref(s), _offsets(offsets, seqs), _dense(h0, h, torch.float32, "h0"), _dense(hT, h, torch.float32, "hT"),
          _states(states, s), wp, wb, _stream())


def sn_scan_bwd(u, dt, A, B, C, D, z, dt_bias, dy, du, ddt, dA, dB, dC, dD, dz, ddt_bias, workspace, offsets=None, seqs=1, h0=None, states=None,
                dhT=None, dh0=None, softplus=True):
    s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, dy, "dy", seqs, softplus, offsets is not None)
    t, gn, vec, h = u.dtype, s.groups * s.states, (s.channels,), (seqs, s.channels, s.states)
    dup, s.ld_du = _rows(du, s.rows, s.channels, t, "du")
    ddtp, s.ld_ddt = _rows(ddt, s.rows, s.channels, t, "ddt")
    dbp, s.ld_db = _rows(dB, s.rows, gn, t, "dB")
    dcp, s.ld_dc = _rows(dC, s.rows, gn, t, "dC")
    dzp, s.ld_dz = _rows(dz, s.rows, s.channels, t, "dz") if dz is not None else (None, 0)
    wp, wb = _bytes(workspace, "workspace")
    _call("sn_scan_bwd", *args, dup, ddtp, _dense(dA, (s.channels, s.states), torch.float32, "dA"), dbp, dcp, _dense(dD, vec, torch.float32, "dD"), dzp,
          _dense(ddt_bias, vec, torch.float32, "ddt_bias"), ctypes.byref(s), _offsets(offsets, seqs), _dense(h0, h, torch.float32, "h0"), _states(states, s),
          _dense(dhT, h, torch.float32, "dhT"), _dense(dh0, h, torch.float32, "dh0"), wp, wb, _stream())


def sn_scan_step(u, dt, A, B, C, D, z, dt_bias, y, state, state_out=None, slots=None, softplus=True):
    """One token for each row of u; state: fp32 (num_slots, channels, states), updated in place unless state_out is given."""
    s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, y, "y", 1, softplus, False)
    shape = (state.shape[0], s.channels, s.states)
    sp = _dense(state, shape, torch.float32, "state")
    _call("sn_scan_step", *args, sp, sp if state_out is None else _dense(state_out, shape, torch.float32, "state_out"), _slots(slots, s.rows), shape[0],
          ctypes.byref(s), _stream())
