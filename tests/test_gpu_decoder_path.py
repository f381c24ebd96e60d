"""The calls between a layer's projections and the next tokens, together as a decoder uses
them: turned and appended, attended to, the head in 8 bits, sampled."""
import importlib.util
import os

import numpy as np
import pytest

from tests import paged
from tests.test_gpu_attn import dev
from tests.test_gpu_rope import turned
from tests.test_gpu_sample import plain
from tests.test_gpu_w8a8 import product, quantized, same

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_prompt_then_steps(pk, layout, cache):
    """Prompts of two sequences, then a step of one token each, in a cache whose keys are
    turned; attention against 64 bits over what the cache holds, head and token exactly."""
    import torch
    g = np.random.default_rng(3)
    H, Hq, D, page, V = 2, 6, 64, 16, 500
    lens = [37, 5]
    T = sum(lens)
    freq, mag = pk.apex4_rope_freq(D, scaling="bands", factor=4.0, trained=64)
    c = pk.PagedKVCache(1, 12, 2, H, D, page, 64, cache)
    assert c.reserved(c.reserve([0, 1], [n + 1 for n in lens]))
    table, _ = c.batch([0, 1])
    start = torch.tensor([0, lens[0], T], dtype=torch.int32, device="cuda")
    qkv = torch.from_numpy(g.standard_normal((T, Hq + 2 * H, D)).astype(np.float16)).cuda()
    q, k, v = torch.split(qkv, [Hq, H, H], dim=1)
    batch = (table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    y = c.prefill(0, c.append_rope(0, q, k, v, batch, freq, start, layout=layout, scale=mag), batch, start, max(lens))
    step = torch.from_numpy(g.standard_normal((2, Hq + 2 * H, D)).astype(np.float16)).cuda()
    q1, k1, v1 = torch.split(step, [Hq, H, H], dim=1)
    batch = (table, torch.tensor([n + 1 for n in lens], dtype=torch.int32, device="cuda"))
    q1r = c.append_rope(0, q1, k1, v1, batch, freq, layout=layout, scale=mag)
    y1 = c.decode(0, q1r, batch)
    # what the cache now holds, from the definition
    for b, n in enumerate(lens):
        at = slice(int(start[b]), int(start[b]) + n)
        pos = np.arange(n + 1)
        both = [torch.cat((x[at], z[b:b + 1])).cpu().numpy() for x, z in ((q, q1), (k, k1), (v, v1))]
        keys, slack = turned(both[1], pos, freq.cpu().numpy(), layout, np.float32(mag).astype(np.float64))
        starts = torch.tensor([0, n + 1], dtype=torch.int32, device="cuda")
        kk, vv = (x.cpu().numpy() for x in pk.apex4_kv_gather(*c.planes[0], table[b:b + 1].contiguous(), batch[1][b:b + 1], n + 1, H, D, page,
                                                             q_start=starts, cache=cache))
        if cache == "fp16":
            assert (np.abs(kk - keys) <= slack).all() and np.array_equal(vv, both[2])
        else:  # a code is half a step off at most, and the scale half a step of binary16
            assert (np.abs(kk - keys) <= (0.5 / 7 + 2.0 ** -8) * np.abs(keys).max(axis=-1, keepdims=True) + slack).all()
        queries = pk.apex4_rope(torch.from_numpy(both[0]).cuda(), dev(pos.astype(np.int32)), freq, layout=layout, scale=mag).cpu().numpy()
        assert np.array_equal(queries[n], q1r[b].cpu().numpy())
        for p in range(n + 1):
            got = (y1[b] if p == n else y[int(start[b]) + p]).cpu().numpy().astype(np.float64)
            # an int4 cache is attended to as codes times scales, not rounded to binary16 as gather's are
            out, mean, top = paged.attention(queries[p], kk.astype(np.float64), vv.astype(np.float64), p, 0, 0, D ** -0.5)
            tol = paged.tolerance(out, mean, top, p + 1)
            if cache == "int4":  # values 2^-11 off, and scores by 2^-11 of sum |q k| / sqrt(D)
                moved = (np.abs(queries[p]).astype(np.float64).reshape(H, -1, D) * np.abs(kk[:p + 1]).max(axis=0)[:, None]).sum(-1).reshape(-1, 1) * D ** -0.5
                tol = tol + mean * (2.0 ** -11 + 2 * np.expm1(moved * 2.0 ** -11))
            assert (np.abs(got - out) <= tol).all()
    # the head and the choice: exact
    w = g.standard_normal((V, Hq * D)).astype(np.float16)
    head = pk.W8A8Linear(dev(w))
    logits = head(y1.view(2, -1))
    qa, sa = quantized(y1.view(2, -1).cpu().numpy())
    qw, sw = quantized(w)
    assert same(logits, product(qa, sa, qw, sw))
    u = np.array([0.3, 0.9], np.float32)
    tokens, probs = pk.apex4_sample(logits, dev(u), temperature=0.9, top_k=40, top_p=0.9, min_p=0.01)
    for b in range(2):
        token, prob, near = plain(logits[b].cpu().numpy(), u[b], np.float32(0.9), 40, np.float32(0.9), np.float32(0.01))
        assert near > 1e-9 and int(tokens[b]) == token and float(probs[b]) == pytest.approx(prob, rel=1e-6)


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serve_layers", os.path.join(ROOT, "examples", "serve_layers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_serving_with_sampled_tokens(example):
    """Runs, gives tokens of the vocabulary, the same again from the same seeds, and other ones
    than the largest logits."""
    import torch
    sizes = dict(layers=2, batch=3, prompt=50, steps=6, hidden=256, heads=4, kv_heads=2, head_dim=64, inner=512, vocab=300,
                 say=lambda *a: None)
    kw = dict(temperature=1.5, top_k=100, top_p=0.95, min_p=0.001)
    a, b, greedy = example.serve(**sizes, **kw), example.serve(**sizes, **kw), example.serve(**sizes)
    assert all(x.equal(y) for x, y in zip(a, b))
    assert all(int(x.min()) >= 0 and int(x.max()) < 300 for x in a)
    assert not torch.equal(a[1], greedy[1])
