"""Python names for the C ABI of include/sn_seq.h (argument marshalling only): layers along token sequences.

Token tensors are torch CUDA (ROCm) tensors of shape (rows, channels), channels contiguous, rows any stride apart; each
call runs on torch's current stream, and its tensors have to live on the current device.  Nothing here computes anything.
"""
import ctypes

import torch

from . import _lib
from .api import SN_BF16, _check, _dtype_code

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
    status = (_fns.get(name) or _fn(name))(*args)
    if status:
        _check(name, status)


# The checks are the larger part of what a small call costs the host: one look at each attribute, messages only when something is wrong.
def _device(t, what):
    """-> the current device, on which t has to live."""
    device = t.get_device()   # below 0: not on a GPU
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError("%s: expected a tensor on the current device" % what)
    return device


def _stream_of(device):
    return torch._C._cuda_getCurrentRawStream(device)


def _refuse(t, shape, dtype, what, device, how):
    if not t.is_cuda or t.get_device() != device:
        raise ValueError("%s: expected a tensor on the current device" % what)
    raise ValueError("%s: expected a %s %s tensor of %s, got %s of %s" % (what, how, tuple(shape), dtype, tuple(t.shape), t.dtype))


def _rows(t, shape, dtype, what, device):
    """-> (pointer, row stride) of a token tensor of that shape."""
    if t.get_device() != device or t.shape != shape or t.dtype is not dtype:
        _refuse(t, shape, dtype, what, device, "two-dimensional")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError("%s: the channels of a row have to be contiguous" % what)
    return t.data_ptr(), ld


def _dense(t, shape, dtype, what, device):
    """-> pointer of a contiguous tensor of that shape, None for None."""
    if t is None:
        return None
    if t.get_device() != device or t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        _refuse(t, shape, dtype, what, device, "contiguous")
    return t.data_ptr()


def _bytes(t, what, device):
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        _refuse(t, t.shape, t.dtype, what, device, "contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


_f32, _int32 = torch.float32, torch.int32


# ---- short causal convolution ----
def _conv1d_shape(x, w, y, what, seqs, silu, dx=None):
    device, t = _device(x, "x"), x.dtype
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x has to be (rows, channels), w (channels, width)")
    shape = x.shape
    rows, channels = shape
    width = w.shape[1]
    xp, ldx = _rows(x, shape, t, "x", device)
    yp, ldy = _rows(y, shape, t, what, device)
    dxp, lddx = _rows(dx, shape, t, "dx", device) if dx is not None else (None, 0)
    wp = _dense(w, (channels, width), t, "w", device)
    return device, xp, wp, yp, dxp, Conv1dShape(rows, seqs, channels, width, 1 if silu else 0, _dtype_code(x), ldx, ldy, lddx)


def sn_causal_conv1d_fwd(x, w, bias, y, offsets=None, seqs=1, state_in=None, state_out=None, silu=True):
    device, xp, wp, yp, _, s = _conv1d_shape(x, w, y, "y", seqs, silu)
    state, t = (seqs, w.shape[1] - 1, w.shape[0]), x.dtype
    _call("sn_causal_conv1d_fwd", xp, wp, _dense(bias, state[2:], _f32, "bias", device), yp, s, _dense(offsets, (seqs + 1,), _int32, "offsets", device),
          _dense(state_in, state, t, "state_in", device), _dense(state_out, state, t, "state_out", device), _stream_of(device))


def sn_causal_conv1d_scratch_bytes(rows, channels, width):
    return int(_fn("sn_causal_conv1d_scratch_bytes")(rows, channels, width))


def sn_causal_conv1d_bwd(x, w, bias, dy, dx, dw, dbias, scratch, offsets=None, seqs=1, state_in=None, dstate_out=None, dstate_in=None, silu=True):
    device, xp, wp, gp, dxp, s = _conv1d_shape(x, w, dy, "dy", seqs, silu, dx)
    state, t = (seqs, w.shape[1] - 1, w.shape[0]), x.dtype
    sp, sb = _bytes(scratch, "scratch", device)
    _call("sn_causal_conv1d_bwd", xp, wp, _dense(bias, state[2:], _f32, "bias", device), gp, dxp, _dense(dw, w.shape, _f32, "dw", device),
          _dense(dbias, state[2:], _f32, "dbias", device), s, _dense(offsets, (seqs + 1,), _int32, "offsets", device),
          _dense(state_in, state, t, "state_in", device), _dense(dstate_out, state, t, "dstate_out", device), _dense(dstate_in, state, t, "dstate_in", device),
          sp, sb, _stream_of(device))


def sn_causal_conv1d_step(x, w, bias, y, state, state_out=None, slots=None, silu=True):
    """One token for each row of x; state: (num_slots, width - 1, channels), updated in place unless state_out is given."""
    device, xp, wp, yp, _, s = _conv1d_shape(x, w, y, "y", 1, silu)
    shape, t = (state.shape[0], w.shape[1] - 1, w.shape[0]), x.dtype
    sp = _dense(state, shape, t, "state", device)
    _call("sn_causal_conv1d_step", xp, wp, _dense(bias, shape[2:], _f32, "bias", device), yp, sp,
          sp if state_out is None else _dense(state_out, shape, t, "state_out", device), _dense(slots, x.shape[:1], _int32, "slots", device), shape[0], s,
          _stream_of(device))


# ---- norm of heads and position rotation ----
def _headnorm_shape(q, k, yq, yk, inv_freq, head_dim, eps, interleaved, dq=None, dk=None):
    if q.dim() != 2 or (k is not None and k.dim() != 2):
        raise ValueError("q and k have to be (rows, heads * head_dim)")
    rows, nq = q.shape
    nk = k.shape[1] if k is not None else 0
    if head_dim < 1 or nq % head_dim or nk % head_dim:
        raise ValueError("the rows of q and k have to hold whole heads of head_dim = %d" % head_dim)
    device, t = _device(q, "q"), q.dtype
    none, sq, sk = (None, 0), (rows, nq), (rows, nk)
    qp, ldq = _rows(q, sq, t, "q", device)
    yqp, ldyq = _rows(yq, sq, t, "yq", device)
    kp, ldk = _rows(k, sk, t, "k", device) if k is not None else none
    ykp, ldyk = _rows(yk, sk, t, "yk", device) if yk is not None else none
    dqp, lddq = _rows(dq, sq, t, "dq", device) if dq is not None else none
    dkp, lddk = _rows(dk, sk, t, "dk", device) if dk is not None else none
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    s = HeadnormShape(rows, nq // head_dim, nk // head_dim, head_dim, rot, 1 if interleaved else 0, _dtype_code(q), eps, ldq, ldk, ldyq, ldyk, lddq, lddk)
    return device, qp, kp, yqp, ykp, dqp, dkp, s


def _headnorm_args(wq, wk, positions, inv_freq, q, head_dim, device):
    return (_dense(wq, (head_dim,), _f32, "wq", device), _dense(wk, (head_dim,), _f32, "wk", device), _dense(positions, q.shape[:1], _int32, "positions", device),
            None if inv_freq is None else _dense(inv_freq, (inv_freq.numel(),), _f32, "inv_freq", device))


def sn_headnorm_rot_fwd(q, k, wq, wk, positions, inv_freq, yq, yk, head_dim, eps=1e-6, interleaved=False):
    """q, k: (rows, heads * head_dim); k and yk may be None.  inv_freq has rot_dim / 2 elements, or is None for no rotation."""
    device, qp, kp, yqp, ykp, _, _, s = _headnorm_shape(q, k, yq, yk, inv_freq, head_dim, eps, interleaved)
    _call("sn_headnorm_rot_fwd", qp, kp, *_headnorm_args(wq, wk, positions, inv_freq, q, head_dim, device), yqp, ykp, s, _stream_of(device))


def sn_headnorm_rot_scratch_bytes(rows, q_heads, k_heads, head_dim):
    return int(_fn("sn_headnorm_rot_scratch_bytes")(rows, q_heads, k_heads, head_dim))


def sn_headnorm_rot_bwd(q, k, wq, wk, positions, inv_freq, dyq, dyk, dq, dk, dwq, dwk, scratch, head_dim, eps=1e-6, interleaved=False):
    device, qp, kp, gqp, gkp, dqp, dkp, s = _headnorm_shape(q, k, dyq, dyk, inv_freq, head_dim, eps, interleaved, dq, dk)
    vec = (head_dim,)
    sp, sb = _bytes(scratch, "scratch", device)
    _call("sn_headnorm_rot_bwd", qp, kp, *_headnorm_args(wq, wk, positions, inv_freq, q, head_dim, device), gqp, gkp, dqp, dkp,
          _dense(dwq, vec, _f32, "dwq", device), _dense(dwk, vec, _f32, "dwk", device), s, sp, sb, _stream_of(device))


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
    if u.dim() != 2 or A.dim() != 2:
        raise ValueError("u has to be (rows, channels), A (channels, states)")
    shape = u.shape
    rows, channels = shape
    states = A.shape[1]
    if states < 1 or B.dim() != 2 or B.shape[1] % states:
        raise ValueError("the rows of B and C have to hold whole groups of states = %d" % states)
    device, t = _device(u, "u"), u.dtype
    vec, bc = (channels,), (rows, B.shape[1])
    up, ldu = _rows(u, shape, t, "u", device)
    dtp, lddt = _rows(dt, shape, t, "dt", device)
    bp, ldb = _rows(B, bc, t, "B", device)
    cp, ldc = _rows(C, bc, t, "C", device)
    zp, ldz = _rows(z, shape, t, "z", device) if z is not None else (None, 0)
    yp, ldy = _rows(y, shape, t, what, device)
    s = ScanShape(rows, seqs, channels, states, bc[1] // states, _dtype_code(u), 1 if softplus else 0, 1 if ragged else 0, ldu, lddt, ldb, ldc, ldz, ldy)
    return device, s, (up, dtp, _dense(A, (channels, states), _f32, "A", device), bp, cp, _dense(D, vec, _f32, "D", device), zp,
                       _dense(dt_bias, vec, _f32, "dt_bias", device), yp)


def _states(states, s, device):
    p, n = _bytes(states, "states", device)
    if states is not None and n < sn_scan_states_bytes(s):
        raise ValueError("states: %d bytes, needs %d" % (n, sn_scan_states_bytes(s)))
    return p


def sn_scan_fwd(u, dt, A, B, C, D, z, dt_bias, y, offsets=None, seqs=1, h0=None, hT=None, states=None, workspace=None, softplus=True):
    """u, dt, z, y: (rows, channels); A: (channels, states); B, C: (rows, groups * states); D, z, dt_bias may be None."""
    device, s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, y, "y", seqs, softplus, offsets is not None)
    h = (seqs, *A.shape)
    wp, wb = _bytes(workspace, "workspace", device)
    _call("sn_scan_fwd", *args, s, _dense(offsets, (seqs + 1,), _int32, "offsets", device), _dense(h0, h, _f32, "h0", device), _dense(hT, h, _f32, "hT", device),
          _states(states, s, device), wp, wb, _stream_of(device))


def sn_scan_bwd(u, dt, A, B, C, D, z, dt_bias, dy, du, ddt, dA, dB, dC, dD, dz, ddt_bias, workspace, offsets=None, seqs=1, h0=None, states=None,
                dhT=None, dh0=None, softplus=True):
    device, s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, dy, "dy", seqs, softplus, offsets is not None)
    t, shape, bc, vec, h = u.dtype, u.shape, B.shape, u.shape[1:], (seqs, *A.shape)
    dup, s.ld_du = _rows(du, shape, t, "du", device)
    ddtp, s.ld_ddt = _rows(ddt, shape, t, "ddt", device)
    dbp, s.ld_db = _rows(dB, bc, t, "dB", device)
    dcp, s.ld_dc = _rows(dC, bc, t, "dC", device)
    dzp, s.ld_dz = _rows(dz, shape, t, "dz", device) if dz is not None else (None, 0)
    wp, wb = _bytes(workspace, "workspace", device)
    _call("sn_scan_bwd", *args, dup, ddtp, _dense(dA, A.shape, _f32, "dA", device), dbp, dcp, _dense(dD, vec, _f32, "dD", device), dzp,
          _dense(ddt_bias, vec, _f32, "ddt_bias", device), s, _dense(offsets, (seqs + 1,), _int32, "offsets", device), _dense(h0, h, _f32, "h0", device),
          _states(states, s, device), _dense(dhT, h, _f32, "dhT", device), _dense(dh0, h, _f32, "dh0", device), wp, wb, _stream_of(device))


def sn_scan_step(u, dt, A, B, C, D, z, dt_bias, y, state, state_out=None, slots=None, softplus=True):
    """One token for each row of u; state: fp32 (num_slots, channels, states), updated in place unless state_out is given."""
    device, s, args = _scan_inputs(u, dt, A, B, C, D, z, dt_bias, y, "y", 1, softplus, False)
    shape = (state.shape[0], *A.shape)
    sp = _dense(state, shape, _f32, "state", device)
    _call("sn_scan_step", *args, sp, sp if state_out is None else _dense(state_out, shape, _f32, "state_out", device),
          _dense(slots, u.shape[:1], _int32, "slots", device), shape[0], s, _stream_of(device))
