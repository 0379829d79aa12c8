"""Binding of linear attention with a decay for each head (``include/linear_attention.h``): argument marshalling only.  Autograd does not see these calls:
results of inputs that require gradients carry none; ``linear_attention_backward`` computes them."""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from .binding import JsError, JS_ERR_ARG, load_library, _elsewhere, _stream_ptr, _there

LA_OK, LA_ERR_INVALID, LA_ERR_CUDA = 0, -1, -2
LA_MAX_D = 128
LA_MAX_T = (1 << 31) - 128
LA_F32, LA_BF16 = 0, 1
_TYPES = {torch.float32: LA_F32, torch.bfloat16: LA_BF16}


class _Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_longlong), ("token", C.c_longlong), ("head", C.c_longlong)]


class _Shape(C.Structure):
    _fields_ = [("type", C.c_int), ("B", C.c_int), ("N", C.c_int), ("T", C.c_longlong), ("H", C.c_int), ("Dk", C.c_int), ("Dv", C.c_int),
                ("cu_seqlens", C.c_void_p), ("log_decay", C.c_void_p), ("scale", C.c_float)]


# the same as bytes: a call of a few microseconds has no time to fill ctypes structures
_tensor_bytes, _shape_bytes = struct.Struct("@Pqqq"), struct.Struct("@iiiqiiiPPf4x")
assert _tensor_bytes.size == C.sizeof(_Tensor) and _shape_bytes.size == C.sizeof(_Shape)
_pack_tensor, _pack_shape = _tensor_bytes.pack, _shape_bytes.pack

_ready = False


def _lib():
    global _ready
    lib = load_library()
    if not _ready:
        vp, sz, sp, tp = C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p        # (structures: bytes)
        lib.la_workspace.argtypes = [sp, C.c_int]
        lib.la_workspace.restype = sz
        lib.la_forward.argtypes = [sp, tp, tp, tp, vp, tp, vp, vp, sz, vp]
        lib.la_backward.argtypes = [sp, tp, tp, tp, vp, tp, vp, tp, tp, tp, vp, vp, sz, vp]
        lib.la_step.argtypes = [sp, tp, tp, tp, vp, tp, vp]
        lib.la_last_error.restype = C.c_char_p
        _ready = True
    return lib


def _bad(what: str):
    raise JsError(JS_ERR_ARG, what)


def _check(rc: int, what: str):
    if rc != LA_OK:
        raise JsError(rc, f"{what}: " + (_lib().la_last_error().decode() if rc == LA_ERR_CUDA else "argument outside the documented limits"))


def _tensor(t, dtype, index, shape, what, written=False):
    if not (t.dtype is dtype and t.get_device() == index and t.shape == shape):
        _bad(f"{what}: expected {shape} of {dtype} on device {index}")
    st = t.stride()
    if shape[-1] > 1 and st[-1] != 1:
        _bad(f"{what}: expected the values of a head side by side")
    if written and not t.is_contiguous() and t.numel() and not _apart(shape, st):
        _bad(f"{what}: its values overlap")
    return _pack_tensor(t.data_ptr(), st[0], st[1] if len(st) == 4 else 0, st[-2])


def _apart(shape, strides):
    """Do a tensor's values lie at places of their own?  (Dimensions in order of stride, each beyond the extent of those before it.)"""
    extent = 1
    for s, n in sorted((s, n) for s, n in zip(strides, shape) if n > 1):
        if s < extent:
            return False
        extent = s * (n - 1) + extent
    return True


def _state(t, shape, index, what):
    if t is None:
        return None
    if not (t.dtype is torch.float32 and t.get_device() == index and t.shape == shape and t.is_contiguous()):
        _bad(f"{what}: expected contiguous float32 {shape} on device {index}")
    return t.data_ptr()


def _shape(q, v, log_decay, scale, cu_seqlens, dims=4):
    """The header's shape, the number of sequences, and q's device."""
    if not (isinstance(q, torch.Tensor) and q.dtype in _TYPES and q.dim() == dims and v.dim() == dims):
        _bad(f"q, v: expected tensors of float32 or bfloat16 with {dims} dimensions")
    index, shape = q.get_device(), q.shape
    if index < 0:
        _bad("q: expected a CUDA tensor")
    H = shape[-2]
    if not (log_decay.dtype is torch.float32 and log_decay.get_device() == index and log_decay.shape == (H,) and log_decay.is_contiguous()):
        _bad(f"log_decay: expected {H} contiguous float32 on device {index}")
    n = B = shape[0]
    N = cu = 0
    if cu_seqlens is not None:
        if not (cu_seqlens.dtype is torch.int32 and cu_seqlens.get_device() == index and cu_seqlens.dim() == 1 and cu_seqlens.is_contiguous()
                and cu_seqlens.shape[0] >= 1):
            _bad(f"cu_seqlens: expected contiguous int32 on device {index}, one more than there are sequences")
        if B != 1:
            _bad("cu_seqlens: packed sequences lie in one row (B = 1)")
        n = N = cu_seqlens.shape[0] - 1
        cu = cu_seqlens.data_ptr()
        if cu == 0:
            _bad("cu_seqlens: no memory")
    s = _pack_shape(_TYPES[q.dtype], B, N, shape[1] if dims == 4 else 1, H, shape[-1], v.shape[-1], cu, log_decay.data_ptr(), scale)
    return s, n, index


def _workspace(s, backward, like):
    n = _lib().la_workspace(s, backward)
    if n == 0:
        _bad(f"sizes outside the documented limits (1 <= Dk, Dv <= {LA_MAX_D}, at most {LA_MAX_T} steps) or a scale that is not finite")
    return like.new_empty((n + 3) // 4), n


def linear_attention(q, k, v, log_decay, scale: float = 1.0, state=None, cu_seqlens=None, need_state: bool = True, out=None, stream=None):
    """Outputs o [B,T,H,Dv] and the states after the last steps [B,H,Dk,Dv] (None unless need_state).

    q, k [B,T,H,Dk], v [B,T,H,Dv] float32 or bfloat16, any strides with a head's values side by side; log_decay [H] float32;
    state [B,H,Dk,Dv] float32: the states to go on from (None: zeros).  cu_seqlens int32 [N+1]: packed sequences (B = 1,
    states [N,H,Dk,Dv]); steps that belong to none of them are left as they are in `out` (undefined without it), which shares no
    memory with the inputs."""
    s, n, index = _shape(q, v, log_decay, scale, cu_seqlens)
    if _elsewhere(index, stream):
        with _there(index, stream):
            return _forward(s, n, index, q, k, v, log_decay, state, need_state, out)
    return _forward(s, n, index, q, k, v, log_decay, state, need_state, out)


def _forward(s, n, index, q, k, v, log_decay, state, need_state, out):
    (B, T, H, Dk), Dv, dtype = q.shape, v.shape[-1], q.dtype
    if out is None:
        out = q.new_empty((B, T, H, Dv))
        to = _pack_tensor(out.data_ptr(), T * H * Dv, H * Dv, Dv)
    else:
        to = _tensor(out, dtype, index, (B, T, H, Dv), "out", True)
    args = [_tensor(t, dtype, index, (B, T, H, d), w) for t, d, w in ((q, Dk, "q"), (k, Dk, "k"), (v, Dv, "v"))]
    s0 = _state(state, (n, H, Dk, Dv), index, "state")
    S = log_decay.new_empty((n, H, Dk, Dv)) if need_state else None
    ws, size = _workspace(s, 0, log_decay)
    _check(_lib().la_forward(s, *args, s0, to, S.data_ptr() if need_state else None, ws.data_ptr(), size, _stream_ptr(None)), "linear_attention")
    return out, S


def linear_attention_backward(q, k, v, log_decay, do, scale: float = 1.0, state=None, dstate=None, cu_seqlens=None, stream=None):
    """Gradients (dq, dk, dv, dstate0) of the loss from its gradients in the outputs (do) and in the last states (dstate, None: zeros).
    The other arguments are those of ``linear_attention``; steps of no sequence get the gradient 0."""
    s, n, index = _shape(q, v, log_decay, scale, cu_seqlens)
    if _elsewhere(index, stream):
        with _there(index, stream):
            return _backward(s, n, index, q, k, v, log_decay, do, state, dstate, cu_seqlens is not None)
    return _backward(s, n, index, q, k, v, log_decay, do, state, dstate, cu_seqlens is not None)


def _backward(s, n, index, q, k, v, log_decay, do, state, dstate, packed):
    (B, T, H, Dk), Dv, dtype = q.shape, v.shape[-1], q.dtype
    ins = [_tensor(t, dtype, index, (B, T, H, d), w) for t, d, w in ((q, Dk, "q"), (k, Dk, "k"), (v, Dv, "v"), (do, Dv, "do"))]
    s0, ds = _state(state, (n, H, Dk, Dv), index, "state"), _state(dstate, (n, H, Dk, Dv), index, "dstate")
    make = q.new_zeros if packed else q.new_empty
    grads = [make((B, T, H, d)) for d in (Dk, Dk, Dv)]
    outs = [_pack_tensor(t.data_ptr(), T * H * d, H * d, d) for t, d in zip(grads, (Dk, Dk, Dv))]
    dS0 = log_decay.new_empty((n, H, Dk, Dv))
    ws, size = _workspace(s, 1, log_decay)
    _check(_lib().la_backward(s, *ins[:3], s0, ins[3], ds, *outs, dS0.data_ptr(), ws.data_ptr(), size, _stream_ptr(None)), "linear_attention_backward")
    return (*grads, dS0)


def linear_attention_step(q, k, v, log_decay, state, scale: float = 1.0, out=None, stream=None):
    """One step: o [B,H,Dv] from q, k [B,H,Dk], v [B,H,Dv]; state [B,H,Dk,Dv] is updated in place."""
    s, n, index = _shape(q, v, log_decay, scale, None, dims=3)
    if state is None:
        _bad("state: the steps' states are needed")
    if _elsewhere(index, stream):
        with _there(index, stream):
            return _step(s, index, q, k, v, state, out)
    return _step(s, index, q, k, v, state, out)


def _step(s, index, q, k, v, state, out):
    (B, H, Dk), Dv, dtype = q.shape, v.shape[-1], q.dtype
    if out is None:
        out = q.new_empty((B, H, Dv))
        to = _pack_tensor(out.data_ptr(), H * Dv, 0, Dv)
    else:
        to = _tensor(out, dtype, index, (B, H, Dv), "out", True)
    _check(_lib().la_step(s, _tensor(q, dtype, index, (B, H, Dk), "q"), _tensor(k, dtype, index, (B, H, Dk), "k"), _tensor(v, dtype, index, (B, H, Dv), "v"),
                          _state(state, (B, H, Dk, Dv), index, "state"), to, _stream_ptr(None)), "linear_attention_step")
    return out
