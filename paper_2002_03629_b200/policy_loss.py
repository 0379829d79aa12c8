"""Binding of the clipped policy loss with its gradient (``include/policy_loss.h``): argument marshalling only."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .adamw import _on, _stream
from .binding import JsError, JS_ERR_ARG, load_library, _stream_ptr

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


def _row(t: Optional[torch.Tensor], N: int, dtype, device, what: str):
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.device == device and t.is_contiguous() and t.dim() == 1 and t.shape[0] == N):
        raise JsError(JS_ERR_ARG, f"{what}: expected {N} contiguous {dtype} on the logits' device")
    return t.data_ptr()


def _matrix(t: torch.Tensor, what: str):
    if not (t.is_cuda and t.dtype in _TYPES and t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1)):
        raise JsError(JS_ERR_ARG, f"{what}: expected a CUDA matrix of float32 or bfloat16 with its columns together")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise JsError(JS_ERR_ARG, f"{what}: rows overlap")
    return t.data_ptr(), max(t.stride(0), t.shape[1])


def policy_loss(logits, actions, old_logp, advantages, weights=None, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, need_grad: bool = True, dlogits=None, stream=None):
    """Loss of every row, logarithm of its action's probability, and the gradient of the summed loss in the logits.

    logits [N, V] float32 or bfloat16; actions [N] int64; old_logp, advantages, weights, ref_logp [N] float32.  weights: each
    row's share of the loss (None: 1 / N), 0 for padding.  dlogits: where the gradient goes (the logits themselves are allowed);
    None makes a new tensor if need_grad.  Returns (loss [N], logp [N], dlogits or None)."""
    z, stride = _matrix(logits, "logits")
    N, V = logits.shape
    dev, f32 = logits.device, torch.float32
    with _on(dev), _stream(stream):
        loss = torch.empty((N,), dtype=f32, device=dev)
        logp = torch.empty_like(loss)
        if dlogits is None and need_grad:
            dlogits = torch.empty((N, V), dtype=logits.dtype, device=dev)
    d, dstride = None, 0
    if dlogits is not None:
        d, dstride = _matrix(dlogits, "dlogits")
        if dlogits.dtype != logits.dtype or dlogits.shape != logits.shape or dlogits.device != dev:
            raise JsError(JS_ERR_ARG, "dlogits: expected the logits' type, shape and device")
    if ref_logp is None and kl_coef != 0.0:
        raise JsError(JS_ERR_ARG, "kl_coef without ref_logp")
    if old_logp is None or advantages is None or actions is None:
        raise JsError(JS_ERR_ARG, "actions, old_logp and advantages are needed")
    with _on(dev):
        rc = _lib().policy_loss(z, _TYPES[logits.dtype], N, V, stride, _row(actions, N, torch.int64, dev, "actions"),
                                _row(old_logp, N, f32, dev, "old_logp"), _row(advantages, N, f32, dev, "advantages"),
                                _row(weights, N, f32, dev, "weights"), _row(ref_logp, N, f32, dev, "ref_logp"), clip_low, clip_high,
                                kl_coef, loss.data_ptr(), logp.data_ptr(), d, dstride, _stream_ptr(stream))
    if rc != PL_OK:
        raise JsError(rc, "policy_loss: " + (_lib().policy_loss_last_error().decode() if rc == PL_ERR_CUDA
                                             else "argument outside the documented limits"))
    return loss, logp, dlogits
