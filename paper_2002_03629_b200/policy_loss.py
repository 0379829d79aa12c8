"""Binding of the clipped policy loss with its gradient (``include/policy_loss.h``): argument marshalling only.  Autograd does not see the call:
loss and logp carry no gradients, ``dlogits`` is the gradient."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import JsError, JS_ERR_ARG, load_library, _elsewhere, _stream_ptr, _there

PL_OK, PL_ERR_INVALID, PL_ERR_CUDA = 0, -1, -2
PL_F32, PL_BF16 = 0, 1
_TYPES = {torch.float32: PL_F32, torch.bfloat16: PL_BF16}

_ready = False


def _lib():
    global _ready
    lib = load_library()
    if not _ready:
        vp, ll, f = C.c_void_p, C.c_longlong, C.c_float
        lib.policy_loss.argtypes = [vp, C.c_int, ll, C.c_int, ll, vp, vp, vp, vp, vp, f, f, f, vp, vp, vp, ll, vp]
        lib.policy_loss_last_error.restype = C.c_char_p
        _ready = True
    return lib


def _row(t: Optional[torch.Tensor], N: int, dtype, index: int, what: str):
    if t is None:
        return None
    if not (t.dtype is dtype and t.get_device() == index and t.shape == (N,) and t.is_contiguous()):
        raise JsError(JS_ERR_ARG, f"{what}: expected {N} contiguous {dtype} on the logits' device")
    return t.data_ptr()


def _matrix(t: torch.Tensor, what: str):
    if not (t.dtype in _TYPES and t.get_device() >= 0 and t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1)):
        raise JsError(JS_ERR_ARG, f"{what}: expected a CUDA matrix of float32 or bfloat16 with its columns together")
    (N, V), row = t.shape, t.stride(0)
    if N > 1 and row < V:
        raise JsError(JS_ERR_ARG, f"{what}: rows overlap")
    return t.data_ptr(), max(row, V)


def policy_loss(logits, actions, old_logp, advantages, weights=None, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, need_grad: bool = True, dlogits=None, stream=None):
    """Loss of every row, logarithm of its action's probability, and the gradient of the summed loss in the logits.

    logits [N, V] float32 or bfloat16; actions [N] int64; old_logp, advantages, weights, ref_logp [N] float32.  weights: each
    row's share of the loss (None: 1 / N), 0 for padding.  dlogits: where the gradient goes (the logits themselves are allowed);
    None makes a new tensor if need_grad.  Returns (loss [N], logp [N], dlogits or None)."""
    index = logits.get_device()
    if index >= 0 and _elsewhere(index, stream):
        with _there(index, stream):
            return policy_loss(logits, actions, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl_coef, need_grad, dlogits)
    z, stride = _matrix(logits, "logits")
    (N, V), f32 = logits.shape, torch.float32
    if ref_logp is None and kl_coef != 0.0:
        raise JsError(JS_ERR_ARG, "kl_coef without ref_logp")
    if old_logp is None or advantages is None or actions is None:
        raise JsError(JS_ERR_ARG, "actions, old_logp and advantages are needed")
    rows = [_row(t, N, f32 if i else torch.int64, index, w) for i, (t, w) in
            enumerate(((actions, "actions"), (old_logp, "old_logp"), (advantages, "advantages"), (weights, "weights"), (ref_logp, "ref_logp")))]
    loss, logp = torch.empty_like(old_logp), torch.empty_like(old_logp)
    d, dstride = None, 0
    if dlogits is None and need_grad:
        dlogits = torch.empty_like(logits, memory_format=torch.contiguous_format)
        d, dstride = dlogits.data_ptr(), V
    elif dlogits is not None:
        d, dstride = _matrix(dlogits, "dlogits")
        if dlogits.dtype is not logits.dtype or dlogits.shape != logits.shape or dlogits.get_device() != index:
            raise JsError(JS_ERR_ARG, "dlogits: expected the logits' type, shape and device")
    rc = _lib().policy_loss(z, _TYPES[logits.dtype], N, V, stride, *rows, clip_low, clip_high, kl_coef, loss.data_ptr(), logp.data_ptr(), d, dstride,
                            _stream_ptr(None))
    if rc != PL_OK:
        raise JsError(rc, "policy_loss: " + (_lib().policy_loss_last_error().decode() if rc == PL_ERR_CUDA
                                             else "argument outside the documented limits"))
    return loss, logp, dlogits
