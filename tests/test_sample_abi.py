"""Refusals of apex4_sample (no GPU needed, nothing launched)."""
import pytest

from tests.test_cache_abi import L, NULL, P, args  # noqa: F401  (L: the fixture)

D = dict(logits=P, type=0, stride=100, B=3, V=100, u=P, temperature=P, temperature_all=1.0, top_k=P, top_k_all=0, top_p=P, top_p_all=1.0,
         min_p=P, min_p_all=0.0, tokens=P, probs=P, workspace=P, workspace_bytes=1 << 12, stream=None)


@pytest.mark.parametrize("bad,rc", [
    (dict(logits=NULL), -1), (dict(u=NULL), -1), (dict(tokens=NULL), -1), (dict(type=2), -2), (dict(type=-1), -2), (dict(B=-1), -2),
    (dict(B=(1 << 21) + 1), -2), (dict(V=0), -2), (dict(V=-1), -2), (dict(V=(1 << 18) + 1, stride=1 << 19), -2), (dict(stride=99), -2),
    (dict(stride=(1 << 40) + 1), -2), (dict(logits=P + 1), -4), (dict(logits=P + 2, type=1), -4), (dict(u=P + 2), -4), (dict(temperature=P + 1), -4), (dict(top_k=P + 2), -4),
    (dict(top_p=P + 3), -4), (dict(min_p=P + 2), -4), (dict(tokens=P + 2), -4), (dict(probs=P + 1), -4), (dict(workspace=P + 8), -4)])
def test_refusals(L, bad, rc):  # noqa: F811
    assert L.apex4_sample(*args(list(D), D, **bad)) == rc


def test_settings_and_probabilities_may_be_left_out(L):  # noqa: F811
    """What is at fault then is a later check (the tokens' alignment)."""
    assert L.apex4_sample(*args(list(D), D, temperature=NULL, top_k=NULL, top_p=NULL, min_p=NULL, probs=NULL, tokens=P + 2)) == -4


def test_size(L):  # noqa: F811
    import ctypes
    b = ctypes.c_int64(-1)
    assert L.apex4_sample_workspace_size(0, 1, 100, None) == -1
    for bad in ((2, 1, 100), (0, -1, 100), (0, (1 << 21) + 1, 100), (1, 1, 0), (1, 1, (1 << 18) + 1)):
        assert L.apex4_sample_workspace_size(*bad, ctypes.byref(b)) == -2
    assert b.value == -1


def test_binding_refuses(L):  # noqa: F811
    import torch

    import paper_2606_08761_amd as pk
    x, u = torch.zeros((2, 8), dtype=torch.float16), torch.zeros(2)
    with pytest.raises(TypeError):  # host tensors: no CPU path
        pk.apex4_sample(x, u)
    with pytest.raises(ValueError):
        pk.apex4_sample(x[0], u)
    for dtype in (torch.bfloat16, torch.int32, "float16"):
        with pytest.raises(TypeError):
            pk.apex4_sample_workspace_size(2, 8, dtype)
