"""The example that runs the linears, the cache and its attention together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serve_layers", os.path.join(ROOT, "examples", "serve_layers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_serve(example, cache, window, sinks):
    import torch
    sizes = dict(layers=2, batch=3, prompt=90, steps=5, cache=cache, window=window, sinks=sinks, hidden=256, heads=4,
                 kv_heads=2, head_dim=64, inner=512, vocab=300, say=lambda *a: None)
    first, tokens, more = example.serve(**sizes)
    assert first.shape == (3,) and tokens.shape == (5, 3) and more.shape == (5, 3)
    assert int(tokens.min()) >= 0 and int(more.max()) < 300
    again = example.serve(**sizes)
    for a, b in zip((first, tokens, more), again):
        assert torch.equal(a, b)


def test_steps_go_on_as_prompts_would(example):
    """A prompt's next token is the one that the steps reach over the same tokens
    (the attention sees the same cache; the linears quantize each token by itself)."""
    import torch
    m = example.Model(layers=1, hidden=256, heads=4, kv_heads=2, head_dim=64, inner=512, vocab=300, slots=2, pages=40,
                      max_len=200)
    g = torch.Generator().manual_seed(3)
    prompt = torch.randint(0, 300, (60,), generator=g).tolist()
    first = m.take_in([prompt], [0])
    tokens = m.decode(first, [0], [60], 4)
    again = m.take_in([prompt + [int(first)]], [1])
    assert int(again) == int(tokens[0, 0])


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_replayed_steps_are_the_eager_ones(example, cache):
    """Every replay of the captured step gives what the step gives uncaptured."""
    import torch
    sizes = dict(layers=2, hidden=256, heads=4, kv_heads=2, head_dim=64, inner=512, vocab=300, slots=3, pages=60, max_len=200, cache=cache)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, 300, (n,), generator=g).tolist() for n in (60, 17, 1)]
    a, b = example.Model(**sizes), example.Model(**sizes)
    first = a.take_in(prompts, [0, 1, 2])
    assert torch.equal(first, b.take_in(prompts, [0, 1, 2]))
    got = a.decode(first, [0, 1, 2], [60, 17, 1], 7)
    assert b.cache.reserved(b.cache.reserve([0, 1, 2], [67, 24, 8]))
    table, _ = b.cache.batch([0, 1, 2])
    lens = torch.tensor([60, 17, 1], dtype=torch.int32, device="cuda")
    current = first
    for i in range(7):
        lens = lens + 1
        current = b.step(current, (table, lens))
        assert torch.equal(current, got[i])
