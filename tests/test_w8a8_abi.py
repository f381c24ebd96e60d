"""Refusals of the 8-bit linears (no GPU needed, nothing launched)."""
import pytest

from tests.test_cache_abi import L, NULL, P, args  # noqa: F401  (L: the fixture)

D = dict(x=P, A_8=P, s_a=P, W_8=P, s_w=P, M=4, N=8, K=64, Y=P, stream=None)
QUANT, GEMM, LINEAR = "x M K A_8 s_a stream".split(), "A_8 s_a W_8 s_w M N K Y stream".split(), "x W_8 s_w M N K Y A_8 s_a stream".split()
CALLS = [("apex4_quantize_act8", QUANT), ("apex4_w8a8_gemm", GEMM), ("apex4_w8a8_linear", LINEAR)]
BAD = [(dict(M=-1), -2), (dict(M=1 << 31), -2), (dict(M=1 << 26, K=64), -2), (dict(K=0), -2), (dict(K=16), -2), (dict(K=48), -2),
       (dict(K=-32), -2), (dict(K=131072), -2), (dict(N=0), -2), (dict(N=-5), -2), (dict(N=1 << 31), -2), (dict(N=1 << 26), -2)]
BAD += [({n: NULL}, -1) for n in ("x", "A_8", "s_a", "W_8", "s_w", "Y")] + [({n: P + 8}, -4) for n in ("x", "A_8", "s_a", "W_8", "s_w", "Y")]


@pytest.mark.parametrize("call,order", CALLS)
@pytest.mark.parametrize("bad,rc", BAD)
def test_refusals(L, call, order, bad, rc):  # noqa: F811
    if set(bad) <= set(order):
        assert getattr(L, call)(*args(order, D, **bad)) == rc


@pytest.mark.parametrize("call,order", CALLS)
def test_no_rows_need_no_row_buffers(L, call, order):  # noqa: F811
    """What is at fault then is a later check: an alignment, or the device."""
    empty = dict(M=0, x=NULL, A_8=NULL, s_a=NULL, Y=NULL)
    assert getattr(L, call)(*args(order, D, **empty)) in (0, -6)
    if "W_8" in order:
        assert getattr(L, call)(*args(order, D, **empty, W_8=P + 4)) == -4


def test_binding_refuses(L):  # noqa: F811
    import torch

    import paper_2606_08761_amd as pk
    x, w, s = torch.zeros((2, 64), dtype=torch.float16), torch.zeros((8, 64), dtype=torch.int8), torch.zeros(8)
    with pytest.raises(TypeError):  # host tensors: no CPU path
        pk.apex4_quantize_act8(x)
    with pytest.raises(TypeError):
        pk.apex4_w8a8_linear(x, w, s)
    with pytest.raises(TypeError):
        pk.W8A8Linear(x)
    for bad in (lambda: pk.apex4_w8a8_linear(x[0], w, s), lambda: pk.apex4_w8a8_linear(x, w[:, :32], s), lambda: pk.apex4_w8a8_linear(x, w, s[:4]),
                lambda: pk.apex4_w8a8_gemm(w, s[:3], w, s), lambda: pk.W8A8Linear(x[0])):
        with pytest.raises(ValueError):
            bad()
