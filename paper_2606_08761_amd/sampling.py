"""Sampling: the binding of ``apex4_sample``.

    tokens, probs = apex4_sample(logits, u, temperature=0.8, top_k=50, top_p=0.95)

A setting is a number for all rows, or a tensor with one for each."""
from __future__ import annotations

import ctypes
import functools

from . import _check, _stream, _torch, lib
from .cache import _one_device, _ptr, _workspace
from .linear8 import _made


def _setting(value, dtype, B, name):
    """(pointer or None, number, tensor or None)."""
    if isinstance(value, _torch().Tensor):
        if tuple(value.shape) != (B,):
            raise ValueError(f"{name} must be a number or [{B}]")
        return _ptr(value, dtype, name), 0, value
    return None, value, None


@functools.lru_cache(maxsize=1024)
def _need(device, type, B, V):
    b = ctypes.c_int64(0)
    _check("apex4_sample_workspace_size", lib().apex4_sample_workspace_size(type, B, V, ctypes.byref(b)))
    return int(b.value)


def apex4_sample_workspace_size(B: int, V: int, dtype) -> int:
    """Bytes of workspace apex4_sample needs for logits [B, V] of dtype on the current device (0: none)."""
    torch = _torch()
    if dtype is not torch.float16 and dtype is not torch.float32:
        raise TypeError("logits must be torch.float16 or torch.float32")
    return _need(torch.cuda.current_device(), 0 if dtype is torch.float16 else 1, B, V)


def apex4_sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, tokens=None, probs=None, workspace=None,
                 stream=None):
    """(tokens int32 [B], probs float32 [B]) of logits [B, V] float16 or float32 (rows any
    distance apart), and random numbers u [B] float32 in [0, 1).  temperature, top_p and
    min_p: numbers or float32 [B]; top_k: a number or int32 [B] (0: off).  A temperature of 0
    takes the largest logit; a row of nothing but -inf gives -1."""
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [B, V]")
    if not logits.is_cuda:
        raise TypeError("logits must be a CUDA (HIP) tensor")
    if logits.dtype is not torch.float16 and logits.dtype is not torch.float32:
        raise TypeError("logits must be torch.float16 or torch.float32")
    B, V = logits.shape
    stride, one = logits.stride()
    if one != 1 and V > 1:
        raise ValueError("the rows of logits must be contiguous")
    if tuple(u.shape) != (B,):
        raise ValueError("u must be [B]")
    tp, t, th = _setting(temperature, torch.float32, B, "temperature")
    kp, k, kh = _setting(top_k, torch.int32, B, "top_k")
    pp, p, ph = _setting(top_p, torch.float32, B, "top_p")
    mp, m, mh = _setting(min_p, torch.float32, B, "min_p")
    tokens = _made(tokens, (B,), torch.int32, logits, stream, "tokens")
    probs = _made(probs, (B,), torch.float32, logits, stream, "probs")
    _one_device(logits, u, th, kh, ph, mh, tokens, probs, workspace)
    kind = 0 if logits.dtype is torch.float16 else 1
    wp, wn, held = _workspace(workspace, _need(logits.get_device(), kind, B, V) if workspace is None else 0, logits, stream)
    rc = lib().apex4_sample(logits.data_ptr(), kind, stride if B > 1 else V, B, V,
                            _ptr(u, torch.float32, "u"), tp, t, kp, k, pp, p, mp, m, _ptr(tokens, torch.int32, "tokens"),
                            _ptr(probs, torch.float32, "probs"), wp, wn, _stream(logits, stream))
    _check("apex4_sample", rc)
    return tokens, probs
