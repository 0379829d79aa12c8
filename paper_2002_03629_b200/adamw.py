"""Binding of the AdamW step (``include/adamw.h``): argument marshalling only.

``adamw_state`` makes the states, ``adamw_step`` updates parameters and states in place on the current stream.
"""
from __future__ import annotations

import ctypes as C
import struct
from itertools import chain
from operator import attrgetter
from typing import NamedTuple, Optional, Sequence, Union

import numpy as np
import torch

from .binding import JsError, JS_ERR_ARG, load_library, _elsewhere, _stream_ptr, _there

ADAMW_OK, ADAMW_ERR_INVALID, ADAMW_ERR_CUDA = 0, -1, -2
ADAMW_BLOCK = 256


class AdamWState(NamedTuple):
    """m and v of all tensors: tensor i's values start at the sum of the sizes before it, each rounded up to a multiple of 256.
    32 bits: float32, scales None.  8 bits: float8_e4m3fn with a float32 scale for every 256 places; v holds its square root."""
    m: torch.Tensor
    v: torch.Tensor
    m_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


class _Options(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", C.c_longlong), ("step_dev", C.c_void_p), ("lr_dev", C.c_void_p), ("grad_scale", C.c_void_p), ("skip", C.c_void_p),
                ("seed", C.c_longlong)]


# the same as bytes (a step over a few small tensors is 4 us of kernel)
_options = struct.Struct("@dddddqPPPPq")
assert _options.size == C.sizeof(_Options)

_ready = False


def _lib():
    global _ready
    lib = load_library()
    if not _ready:
        vp = C.c_void_p
        lib.adamw_step.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, vp, vp, vp, vp, vp]
        lib.adamw_last_error.restype = C.c_char_p
        _ready = True
    return lib


def _bad(what: str):
    raise JsError(JS_ERR_ARG, what)


def _places(sizes):
    return sum((n + ADAMW_BLOCK - 1) // ADAMW_BLOCK * ADAMW_BLOCK for n in sizes)


def adamw_state(params: Sequence[torch.Tensor], bits: int = 32) -> AdamWState:
    """States of zeros for these parameters, on their device."""
    if bits not in (32, 8):
        _bad("bits: 32 or 8")
    if not params:
        _bad("params: no tensors")
    n, device = _places([p.numel() for p in params]), params[0].device
    if bits == 32:
        return AdamWState(torch.zeros(n, dtype=torch.float32, device=device), torch.zeros(n, dtype=torch.float32, device=device))
    m, v = (torch.zeros(n, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.full((n // ADAMW_BLOCK,), 2.0 ** -120, dtype=torch.float32, device=device) for _ in range(2))
    return AdamWState(m, v, ms, vs)


_numel, _data_ptr, _get_device, _contiguous = torch.Tensor.numel, torch.Tensor.data_ptr, torch.Tensor.get_device, torch.Tensor.is_contiguous
_dtype = attrgetter("dtype")


def _same(tensors, dtype, index, sizes, what: str):
    """Are all of one type, on one device, contiguous, of these sizes?"""
    if (set(map(_dtype, tensors)) != {dtype} or set(map(_get_device, tensors)) != {index} or not all(map(_contiguous, tensors))
            or (sizes is not None and list(map(_numel, tensors)) != sizes)):
        _bad(f"{what}: expected contiguous tensors of {dtype}, of the parameters' sizes and on their device")


def _one(t, dtype, device, what):
    if t is None:
        return None
    if not (t.is_cuda and t.dtype is dtype and t.numel() == 1 and t.device == device):
        _bad(f"{what}: expected one {dtype} on the parameters' device")
    return t.data_ptr()


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], state: AdamWState, step: Union[int, torch.Tensor],
               lr: Union[float, torch.Tensor], betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
               copies: Optional[Sequence[torch.Tensor]] = None, grad_scale: Optional[torch.Tensor] = None,
               skip: Optional[torch.Tensor] = None, seed: Optional[int] = None, stream=None) -> None:
    """One step on all tensors, in place (parameters that require gradients too: autograd is told nothing of it).

    params      float32, contiguous, no two the same; grads of the same sizes, all float32 or all bfloat16, contiguous
    state       from ``adamw_state`` (or a tuple laid out like it)
    step        number of the step, 1 or more; or an int64 tensor on the device, which a captured call reads anew at every replay
    lr          learning rate; or a float32 tensor on the device
    copies      bfloat16 tensors that take the new parameters rounded, for the next forward pass
    grad_scale  one float32 on the device: factor of all gradients
    skip        one int32 on the device: not zero leaves everything as it is (a step whose gradients overflowed)
    seed        of the random roundings of 8-bit states (the step's number if None)
    """
    n = len(params)
    m, v, m_scale, v_scale = state
    if len(grads) != n or (copies is not None and len(copies) != n):
        _bad("params, grads and copies: as many tensors of each")
    if n == 0:
        return
    device, f32 = params[0].device, torch.float32
    if device.type != "cuda":
        _bad("params: expected CUDA tensors")
    # (the checks of many tensors go through C functions mapped over the lists: a step over 300 tensors is 300 us of kernels)
    index, gtype = device.index, grads[0].dtype
    if gtype is not f32 and gtype is not torch.bfloat16:
        _bad("grads: expected float32 or bfloat16")
    sizes, pointers = list(map(_numel, params)), list(map(_data_ptr, params))
    _same(params, f32, index, None, "params")
    _same(grads, gtype, index, sizes, "grads")
    if copies is not None:
        _same(copies, torch.bfloat16, index, sizes, "copies")
    bits = 32 if m.dtype is f32 else 8
    # the header's table of tensors, parameter, gradient, copy, size: packed as bytes; many of them array by array and turned (300: 16 us for 31)
    columns = (pointers, list(map(_data_ptr, grads)), [0] * n if copies is None else list(map(_data_ptr, copies)), sizes)
    if n <= 32:
        table, blocks = struct.pack("@%dq" % (4 * n), *chain.from_iterable(zip(*columns))), sum([(k + (ADAMW_BLOCK - 1)) // ADAMW_BLOCK for k in sizes])
    else:
        turned = np.frombuffer(struct.pack("@%dq" % (4 * n), *chain.from_iterable(columns)), dtype=np.int64).reshape(4, n)
        table, blocks = turned.T.tobytes(), int(((turned[3] + (ADAMW_BLOCK - 1)) // ADAMW_BLOCK).sum())
    stype, places = (f32 if bits == 32 else torch.float8_e4m3fn), blocks * ADAMW_BLOCK
    for t, what in ((m, "m"), (v, "v")):
        if not (t.dtype is stype and t.get_device() == index and t.is_contiguous() and t.numel() == places):
            _bad(f"state.{what}: expected {places} contiguous values of {stype} on the parameters' device")
    if bits == 8:
        for t, what in ((m_scale, "m_scale"), (v_scale, "v_scale")):
            if not (t is not None and t.dtype is f32 and t.get_device() == index and t.is_contiguous() and t.numel() == places // ADAMW_BLOCK):
                _bad(f"state.{what}: expected {places // ADAMW_BLOCK} contiguous float32 on the parameters' device")
    live = pointers if 0 not in sizes else [a for a, k in zip(pointers, sizes) if k]
    if len(set(live)) != len(live):
        _bad("params: the same tensor twice")
    step_dev = lr_dev = None
    if isinstance(step, torch.Tensor):
        step, step_dev = 0, _one(step, torch.int64, device, "step")
    if isinstance(lr, torch.Tensor):
        lr, lr_dev = 0.0, _one(lr, f32, device, "lr")
    o = _options.pack(lr, betas[0], betas[1], eps, weight_decay, int(step), step_dev or 0, lr_dev or 0, _one(grad_scale, f32, device, "grad_scale") or 0,
                      _one(skip, torch.int32, device, "skip") or 0, -1 if seed is None else int(seed) & 0xFFFFFFFF)
    args = (table, n, 0 if gtype is f32 else 1, bits, m.data_ptr(), v.data_ptr(), m_scale.data_ptr() if bits == 8 else None,
            v_scale.data_ptr() if bits == 8 else None, o)
    if _elsewhere(index, stream):
        with _there(index, stream):
            rc = _lib().adamw_step(*args, _stream_ptr(None))
    else:
        rc = _lib().adamw_step(*args, _stream_ptr(None))
    if rc != ADAMW_OK:
        raise JsError(rc, "adamw_step: " + (_lib().adamw_last_error().decode() if rc == ADAMW_ERR_CUDA else "argument outside the documented limits"))
