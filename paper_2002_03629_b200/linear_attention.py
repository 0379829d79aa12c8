"""Binding of linear attention with a decay for each head (``include/linear_attention.h``): argument marshalling only."""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional

import torch

from .adamw import _on, _stream
from .binding import JsError, JS_ERR_ARG, load_library, _stream_ptr

LA_OK, LA_ERR_INVALID, LA_ERR_CUDA, LA_ERR_TIMEOUT = 0, -1, -2, -3
LA_MAX_D = 128
LA_F32, LA_BF16 = 0, 1
_TYPES = {torch.float32: LA_F32, torch.bfloat16: LA_BF16}


class _Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_longlong), ("token", C.c_longlong), ("head", C.c_longlong)]


class _Shape(C.Structure):
    _fields_ = [("type", C.c_int), ("B", C.c_int), ("N", C.c_int), ("T", C.c_longlong), ("H", C.c_int), ("Dk", C.c_int), ("Dv", C.c_int),
                ("cu_seqlens", C.c_void_p), ("log_decay", C.c_void_p), ("scale", C.c_float)]


_ready = False


def _lib():
    global _ready
    lib = load_library()
    if not _ready:
        vp, sz, sp, tp = C.c_void_p, C.c_size_t, C.POINTER(_Shape), C.POINTER(_Tensor)
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


def _tensor(t, like, shape, what, written=False):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == like.dtype and t.device == like.device and t.shape == shape):
        _bad(f"{what}: expected {tuple(shape)} of {like.dtype} on {like.device}")
    st = t.stride()
    if shape[-1] > 1 and st[-1] != 1:
        _bad(f"{what}: expected the values of a head side by side")
    if written and t.numel() and not _apart(shape, st):
        _bad(f"{what}: its values overlap")
    return _Tensor(t.data_ptr(), st[0], st[1] if len(shape) == 4 else 0, st[-2])


def _apart(shape, strides):
    """Do a tensor's values lie at places of their own?  (Dimensions in order of stride, each beyond the extent of those before it.)"""
    extent = 1
    for s, n in sorted((s, n) for s, n in zip(strides, shape) if n > 1):
        if s < extent:
            return False
        extent = s * (n - 1) + extent
    return True


def _state(t, shape, device, what):
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == torch.float32 and t.device == device and t.shape == shape and t.is_contiguous()):
        _bad(f"{what}: expected contiguous float32 {tuple(shape)} on {device}")
    return t.data_ptr()


def _shape(q, k, v, log_decay, scale, cu_seqlens, dims=4):
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dtype in _TYPES and q.dim() == dims):
        _bad(f"q: expected a CUDA tensor of float32 or bfloat16 with {dims} dimensions")
    if v.dim() != dims:
        _bad(f"v: expected {dims} dimensions")
    H, Dk, Dv, device = q.shape[-2], q.shape[-1], v.shape[-1], q.device
    if not (log_decay.is_cuda and log_decay.dtype == torch.float32 and log_decay.device == device and log_decay.shape == (H,)
            and log_decay.is_contiguous()):
        _bad(f"log_decay: expected {H} contiguous float32 on {device}")
    s = _Shape(type=_TYPES[q.dtype], B=q.shape[0], N=0, T=q.shape[1] if dims == 4 else 1, H=H, Dk=Dk, Dv=Dv, log_decay=log_decay.data_ptr(),
               scale=scale)
    n = q.shape[0]
    if cu_seqlens is not None:
        if not (cu_seqlens.is_cuda and cu_seqlens.dtype == torch.int32 and cu_seqlens.device == device and cu_seqlens.dim() == 1
                and cu_seqlens.is_contiguous() and cu_seqlens.shape[0] >= 1):
            _bad(f"cu_seqlens: expected contiguous int32 on {device}, one more than there are sequences")
        if q.shape[0] != 1:
            _bad("cu_seqlens: packed sequences lie in one row (B = 1)")
        n = cu_seqlens.shape[0] - 1
        s.N, s.cu_seqlens = n, cu_seqlens.data_ptr()
    return s, n


def _workspace(s, backward, device):
    n = _lib().la_workspace(C.byref(s), backward)
    if n == 0:
        _bad(f"sizes outside the documented limits (1 <= Dk, Dv <= {LA_MAX_D})")
    return torch.empty((n,), dtype=torch.uint8, device=device), n


def linear_attention(q, k, v, log_decay, scale: float = 1.0, state=None, cu_seqlens=None, need_state: bool = True, out=None, stream=None):
    """Outputs o [B,T,H,Dv] and the states after the last steps [B,H,Dk,Dv] (None unless need_state).

    q, k [B,T,H,Dk], v [B,T,H,Dv] float32 or bfloat16, any strides with a head's values side by side; log_decay [H] float32;
    state [B,H,Dk,Dv] float32: the states to go on from (None: zeros).  cu_seqlens int32 [N+1]: packed sequences (B = 1,
    states [N,H,Dk,Dv]); steps that belong to none of them are left as they are in `out` (undefined without it)."""
    s, n = _shape(q, k, v, log_decay, scale, cu_seqlens)
    B, T, H, Dk = q.shape
    Dv, dev = v.shape[-1], q.device
    with _on(dev), _stream(stream):
        if out is None:
            out = torch.empty((B, T, H, Dv), dtype=q.dtype, device=dev)
        args = [_tensor(t, q, (B, T, H, d), w, w == "out") for t, d, w in ((q, Dk, "q"), (k, Dk, "k"), (v, Dv, "v"), (out, Dv, "out"))]
        s0 = _state(state, (n, H, Dk, Dv), dev, "state")
        S = torch.empty((n, H, Dk, Dv), dtype=torch.float32, device=dev) if need_state else None
        ws, size = _workspace(s, 0, dev)
        _check(_lib().la_forward(C.byref(s), *map(C.byref, args[:3]), s0, C.byref(args[3]), S.data_ptr() if need_state else None, ws.data_ptr(), size,
                                 _stream_ptr(stream)), "linear_attention")
    return out, S


def linear_attention_backward(q, k, v, log_decay, do, scale: float = 1.0, state=None, dstate=None, cu_seqlens=None, stream=None):
    """Gradients (dq, dk, dv, dstate0) of the loss from its gradients in the outputs (do) and in the last states (dstate, None: zeros).
    The other arguments are those of ``linear_attention``; steps of no sequence get the gradient 0."""
    s, n = _shape(q, k, v, log_decay, scale, cu_seqlens)
    B, T, H, Dk = q.shape
    Dv, dev = v.shape[-1], q.device
    ins = [_tensor(t, q, (B, T, H, d), w) for t, d, w in ((q, Dk, "q"), (k, Dk, "k"), (v, Dv, "v"), (do, Dv, "do"))]
    s0, ds = _state(state, (n, H, Dk, Dv), dev, "state"), _state(dstate, (n, H, Dk, Dv), dev, "dstate")
    with _on(dev), _stream(stream):
        make = torch.empty if cu_seqlens is None else torch.zeros
        grads = [make((B, T, H, d), dtype=q.dtype, device=dev) for d in (Dk, Dk, Dv)]
        outs = [_tensor(t, q, t.shape, "gradient") for t in grads]
        dS0 = torch.empty((n, H, Dk, Dv), dtype=torch.float32, device=dev)
        ws, size = _workspace(s, 1, dev)
        _check(_lib().la_backward(C.byref(s), *map(C.byref, ins[:3]), s0, C.byref(ins[3]), ds, *map(C.byref, outs), dS0.data_ptr(), ws.data_ptr(),
                                  size, _stream_ptr(stream)), "linear_attention_backward")
    return (*grads, dS0)


def linear_attention_step(q, k, v, log_decay, state, scale: float = 1.0, out=None, stream=None):
    """One step: o [B,H,Dv] from q, k [B,H,Dk], v [B,H,Dv]; state [B,H,Dk,Dv] is updated in place."""
    s, n = _shape(q, k, v, log_decay, scale, None, dims=3)
    B, H, Dk = q.shape
    Dv, dev = v.shape[-1], q.device
    if state is None:
        _bad("state: the steps' states are needed")
    with _on(dev), _stream(stream):
        if out is None:
            out = torch.empty((B, H, Dv), dtype=q.dtype, device=dev)
    args = [_tensor(t, q, (B, H, d), w, w == "out") for t, d, w in ((q, Dk, "q"), (k, Dk, "k"), (v, Dv, "v"), (out, Dv, "out"))]
    st = _state(state, (B, H, Dk, Dv), dev, "state")
    with _on(dev):
        _check(_lib().la_step(C.byref(s), *map(C.byref, args[:3]), st, C.byref(args[3]), _stream_ptr(stream)), "linear_attention_step")
    return out
