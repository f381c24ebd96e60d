"""Linears in 8 bits, one scale a token and one a channel: bindings of
``apex4_quantize_act8`` and the ``apex4_w8a8_*`` calls of include/apex4.h, and the layer
``W8A8Linear`` for where 4 bits are too few (an output head, a sensitive projection).

    W_8, s_w = apex4_quantize_act8(w)         # w: [N, K] float16 on cuda
    Y = apex4_w8a8_linear(x, W_8, s_w)        # x: [M, K] float16 -> [M, N] float16
    lin = W8A8Linear(w); y = lin(x)           # the same as a layer
"""
from __future__ import annotations

from . import _check, _stream, _torch, lib
from .cache import _empty, _one_device, _output, _ptr


def _made(t, shape, dtype, like, stream, name):
    if t is None:
        return _empty(like, shape, dtype, stream)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}")
    return t


def _matrix(t, name):
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    return t.shape


def _weights(W_8, s_w, K):
    shape = _matrix(W_8, "W_8")
    if shape[1] != K or s_w.shape != shape[:1]:
        raise ValueError(f"W_8 must be [N, {K}] and s_w [N]")
    return shape[0]


def apex4_quantize_act8(x, A_8=None, s_a=None, stream=None):
    """Codes int8 [M, K] and scales float32 [M] of x [M, K] float16, a scale a row."""
    torch = _torch()
    M, K = _matrix(x, "x")
    xp = _ptr(x, torch.float16, "x")
    A_8 = _made(A_8, (M, K), torch.int8, x, stream, "A_8")
    s_a = _made(s_a, (M,), torch.float32, x, stream, "s_a")
    _one_device(x, A_8, s_a)
    rc = lib().apex4_quantize_act8(xp, M, K, _ptr(A_8, torch.int8, "A_8"), _ptr(s_a, torch.float32, "s_a"), _stream(x, stream))
    _check("apex4_quantize_act8", rc)
    return A_8, s_a


def apex4_w8a8_gemm(A_8, s_a, W_8, s_w, Y=None, stream=None):
    """Y [M, N] float16 = s_a s_w^T (.) (A_8 W_8^T) of int8 codes [M, K] and [N, K]."""
    torch = _torch()
    M, K = _matrix(A_8, "A_8")
    N = _weights(W_8, s_w, K)
    if tuple(s_a.shape) != (M,):
        raise ValueError("s_a must be [M]")
    Ap = _ptr(A_8, torch.int8, "A_8")
    Y = _output(Y, (M, N), A_8, stream)
    _one_device(A_8, s_a, W_8, s_w, Y)
    rc = lib().apex4_w8a8_gemm(Ap, _ptr(s_a, torch.float32, "s_a"), _ptr(W_8, torch.int8, "W_8"), _ptr(s_w, torch.float32, "s_w"),
                               M, N, K, _ptr(Y, torch.float16, "Y"), _stream(A_8, stream))
    _check("apex4_w8a8_gemm", rc)
    return Y


def apex4_w8a8_linear(x, W_8, s_w, Y=None, A_8_work=None, s_a_work=None, stream=None):
    """apex4_quantize_act8 of x [M, K] float16, then apex4_w8a8_gemm, in one call; the work
    buffers (made here when None) are scratch."""
    torch = _torch()
    M, K = _matrix(x, "x")
    N = _weights(W_8, s_w, K)
    xp = _ptr(x, torch.float16, "x")
    _one_device(x, W_8, s_w, Y, A_8_work, s_a_work)
    Y = _output(Y, (M, N), x, stream)
    if A_8_work is None and s_a_work is None:  # one buffer for both: an allocation is 1.5 us of a small call's 12
        work = _empty(x, (M * (K + 4),), torch.uint8, stream)
        Ap = work.data_ptr()
        sp = Ap + M * K
    else:
        A_8_work = _made(A_8_work, (M, K), torch.int8, x, stream, "A_8_work")
        s_a_work = _made(s_a_work, (M,), torch.float32, x, stream, "s_a_work")
        Ap, sp = _ptr(A_8_work, torch.int8, "A_8_work"), _ptr(s_a_work, torch.float32, "s_a_work")
    rc = lib().apex4_w8a8_linear(xp, _ptr(W_8, torch.int8, "W_8"), _ptr(s_w, torch.float32, "s_w"), M, N, K,
                                 _ptr(Y, torch.float16, "Y"), Ap, sp, _stream(x, stream))
    _check("apex4_w8a8_linear", rc)
    return Y


class W8A8Linear:
    """A linear layer in 8 bits beside ``W4A4Linear``: the fp16 weight [N, K] is quantized
    once (a scale a channel), and every forward quantizes the fp16 activations (a scale a
    token) and runs the product.

        lin = W8A8Linear(weight_fp16_cuda)
        y = lin(x)             # x [..., K] float16 on the same device -> [..., N]

    The work buffers of a call belong to its stream, so forwards on different streams
    never share them."""

    def __init__(self, weight):
        if weight.dim() != 2:
            raise ValueError("weight must be [N, K]")
        self.N, self.K = weight.shape
        self.W_8, self.s_w = apex4_quantize_act8(weight.contiguous())

    def __call__(self, x, stream=None):
        if x.shape[-1] != self.K:
            raise ValueError(f"expected last dimension {self.K}, got {x.shape[-1]}")
        shape = x.shape[:-1]
        if not x.is_contiguous():
            with _torch().cuda.stream(stream):  # None: the current one
                x = x.contiguous()
        if len(shape) == 1:
            return apex4_w8a8_linear(x, self.W_8, self.s_w, stream=stream)
        return apex4_w8a8_linear(x.view(-1, self.K), self.W_8, self.s_w, stream=stream).view(*shape, self.N)
