"""Sampling against the definition in 80 bits, and where the outcome is known without
arithmetic."""
import numpy as np
import pytest

from tests.test_gpu_attn import dev

pytestmark = pytest.mark.gpu
F32 = np.float32


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def plain(x, u, t, k, p, least):
    """(token, probability, how near the decision was: the distance of u's target from the
    borders of the token's share, and of top-p's from the running sums beside it, as shares)."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.longdouble))
    order = np.argsort(-x, kind="stable")
    if not x[order[0]] > -np.inf:
        return -1, 0.0, 1.0
    if not t > 0 or k == 1 or p <= 0 or least > 1:
        return int(order[0]), 1.0, 1.0
    d = np.where(x == x[order[0]], 0, x - x[order[0]])
    with np.errstate(invalid="ignore"):
        w = np.where(d == 0, 1, np.exp(np.where(d == -np.inf, -np.inf, d / np.longdouble(t))))
    s = w[order]
    n, near = len(x), 1.0
    if 0 < k < n:
        n = k
    if p < 1:
        run = np.cumsum(s[:n])
        cut = np.longdouble(p) * run[-1]
        near = float(np.abs(run - cut).min() / run[-1])
        n = min(n, int((run < cut).sum()) + 1)
    if least > 0:
        inside = s[:n] >= np.longdouble(least)
        n = max(1, int(inside.sum()))
    chosen = np.sort(order[:n])
    run = np.cumsum(w[chosen])
    goal = np.longdouble(min(max(float(u), 0.0), 1.0) if u == u else 0.0) * run[-1]
    i = int((run <= goal).sum())
    if i >= len(chosen) or u >= 1:
        i = int(np.nonzero(w[chosen] > 2.0 ** -45)[0][-1])
    if u < 1:
        near = min(near, float(np.abs(run[max(0, i - 1):i + 1] - goal).min() / run[-1]) if goal > 0 else 1.0)
    return int(chosen[i]), float(w[chosen[i]] / run[-1]), near


def check(pk, x, u, t=1.0, k=0, p=1.0, least=0.0, gap=0):
    """x [B, V]; settings: numbers or [B].  Rounded weights (2^-46 of the largest each, V of
    them) decide otherwise than exact ones only where a decision is as near as that."""
    import torch
    B, V = x.shape
    wide = np.zeros((B, V + gap), x.dtype)
    wide[:, :V] = x
    u = np.asarray(u, F32)
    kw = {n: dev(np.asarray(v, np.int32 if n == "top_k" else F32)) if np.ndim(v) else v
          for n, v in (("temperature", t), ("top_k", k), ("top_p", p), ("min_p", least))}
    tokens, probs = (y.cpu().numpy() for y in pk.apex4_sample(dev(wide)[:, :V], dev(u), **kw))
    assert torch.cuda.current_stream() is not None
    full = [np.broadcast_to(np.asarray(v, np.int64 if n == "k" else F32), (B,)) for n, v in (("t", t), ("k", k), ("p", p), ("least", least))]
    for b in range(B):
        token, prob, near = plain(x[b], u[b], *(f[b] for f in full))
        assert tokens[b] == token or near <= V * 2.0 ** -45, (b, tokens[b], token, near)
        if tokens[b] == token:  # probabilities: binary64 quotients, rounded to binary32; the sum is off by V units
            assert abs(probs[b] - prob) <= 2.0 ** -24 * prob + V * 2.0 ** -45 + 1e-45, (b, probs[b], prob)


def logits(g, B, V, dtype, sd=2.0):
    return (g.standard_normal((B, V)) * sd + 10 * g.random((B, V)) ** 300).astype(dtype)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 1000, 1025, 16383, 32000, 32001, 32768, 65535, 100003, 131072, 262144])
def test_every_setting(pk, dtype, V):
    g = np.random.default_rng(V)
    B = 12 if V < 40000 else 6
    x = logits(g, B, V, dtype)
    u = g.random(B)
    t = (0.5 + g.random(B)).astype(F32)
    check(pk, x, u)
    check(pk, x, u, t=t, p=(0.5 + 0.5 * g.random(B)).astype(F32))
    check(pk, x, u, t=t, k=g.integers(0, 200, B))
    check(pk, x, u, t=0.7, k=max(2, V // 3), p=0.9, gap=13)
    check(pk, x, u, t=t, least=(0.2 * g.random(B)).astype(F32))
    check(pk, x, u, t=t, k=40, p=0.95, least=0.01, gap=3)
    check(pk, x, u, t=np.where(np.arange(B) % 3 == 0, 0, t), k=np.where(np.arange(B) % 2 == 0, 0, 50), p=np.where(np.arange(B) % 4 == 1, 1, 0.8).astype(F32),
          least=np.where(np.arange(B) % 5 == 0, 0.1, 0).astype(F32))


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("V", [5, 1000, 32000, 90001, 262144])
def test_equal_logits(pk, dtype, V):
    """n equal ones are kept, the lowest indexes: the token is floor(u n).  (More members of a
    bucket than its list holds.)"""
    import torch
    B = 16
    g = np.random.default_rng(V)
    x = torch.full((B, V), 3.25, dtype=torch.float16 if dtype == np.float16 else torch.float32, device="cuda")
    u = g.random(B).astype(F32)
    u[:3] = [0.0, 1 - 2.0 ** -24, 0.5]

    def tokens(n, **kw):
        got, probs = pk.apex4_sample(x, dev(u), **kw)
        assert np.array_equal(got.cpu().numpy(), [int(float(v) * n) for v in u.astype(np.float64)])
        assert np.array_equal(probs.cpu().numpy(), np.full(B, 1 / n, F32))
    tokens(V)
    tokens(V, temperature=0.3, min_p=1.0)
    for k in {2, max(2, V // 2), max(2, V - 1), V, V + 5}:
        tokens(min(k, V), top_k=k)
    for p in (0.25, 0.5, 0.75):  # exact in binary: ceil(p V) of them
        tokens(int(np.ceil(p * V)), top_p=p)
        tokens(int(np.ceil(p * max(2, V // 2))), top_p=p, top_k=max(2, V // 2))


def test_two_values(pk):
    """Ties on both sides of the border, spread over the row."""
    import torch
    g = np.random.default_rng(3)
    for V in (3000, 50000):
        high = g.permutation(V)[:V // 5]
        x = np.full((1, V), 1.0, np.float16)
        x[0, high] = 2.0
        low = np.setdiff1d(np.arange(V), high)
        for extra in (1, 2, 257, len(low) - 1):
            keep = np.sort(np.concatenate((high, np.sort(low)[:extra])))
            e = np.exp(-1.0)
            w = np.where(np.isin(keep, high), 1.0, e)
            for u in (0.0, 0.3, 0.9999, 1 - 2.0 ** -24):
                want = keep[(np.cumsum(w) <= F32(u) * w.sum()).sum()]
                got, _ = pk.apex4_sample(dev(x), torch.tensor([u], device="cuda"), top_k=len(high) + extra)
                assert int(got) == want
                # a share in the midst of the extra-th one's weight keeps as many
                share = (len(high) + (extra - 0.5) * e) / (len(high) + len(low) * e)
                got, _ = pk.apex4_sample(dev(x), torch.tensor([u], device="cuda"), top_p=float(F32(share)))
                assert int(got) == want


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("B,V", [(9, 700), (9, 32000), (30, 70001), (2, 70001)])
def test_top_p_of_a_small_top_k(pk, B, V, dtype):
    """As many logits as top-k keeps, fewer, and more equal ones at its border than a list holds."""
    import torch
    g = np.random.default_rng(V + B)
    x = logits(g, B, V, dtype)
    u = g.random(B)
    for k in (2, 50, 600, 1024, 1025):
        for p in (0.2, 0.9):
            check(pk, x, u, k=k, p=p)
            check(pk, x, u, k=k, p=p, t=1.7, least=0.02)
    some = x.copy()
    some[:, 40:] = -np.inf
    check(pk, some, u, k=50, p=0.8)
    check(pk, some, u, k=40, p=0.8)
    check(pk, some, u, k=39, p=0.8)
    flat = torch.full((B, V), 0.5, dtype=torch.float16 if dtype == np.float16 else torch.float32, device="cuda")
    flat[:, 5] = 0.5 + np.log(8.0)  # not exact: its share is near 8
    got, _ = pk.apex4_sample(flat, dev(u.astype(F32)), top_k=401, top_p=0.5)
    assert ((got >= 0) & (got <= 198)).all()  # 8 and 400 ones: 196 ones, up to a rounding of the logit
    got, _ = pk.apex4_sample(flat, torch.full((B,), 1 - 2.0 ** -24, device="cuda"), top_k=401, top_p=0.5)
    assert ((got >= 194) & (got <= 198)).all()


@pytest.mark.parametrize("B,V,dtype", [(14, 32000, np.float16), (14, 31999, np.float32), (24, 70001, np.float32), (3, 70001, np.float16)])
def test_top_p_and_min_p_together(pk, B, V, dtype):
    """min-p's border behind top-p's, beside it in the same bucket, and before it; tokens in
    every part of the row."""
    g = np.random.default_rng(V)
    x = (g.standard_normal((B, V)) * 1.5).astype(dtype)
    u = ((np.arange(B) + g.random(B)) / B).astype(F32)
    for p in (0.3, 0.8, 0.97):
        w = np.sort(np.exp((x[0] - x[0].max()).astype(np.float64)))[::-1]
        border = w[(np.cumsum(w) < p * w.sum()).sum()]
        for near in (1e-3, 0.5, 0.97, 0.999, 1.001, 1.03, 2.0, 30.0):
            check(pk, x, u, p=p, least=border * near)


@pytest.mark.parametrize("V", [600, 50001, 131072])
def test_borders_at_zero(pk, V):
    """Zeros of both signs are one value, at the border, above it and as the largest."""
    import torch
    g = np.random.default_rng(V)
    sign = np.where(g.random(V) < 0.5, 0.0, -0.0)
    for other in (1.0, -1.0):
        x = np.where(np.arange(V) % 3 == 0, other, sign).astype(np.float32)[None]
        for u in (0.0, 0.7, 1 - 2.0 ** -24):
            for kw in (dict(), dict(top_k=V // 3 + 100), dict(top_k=V // 2), dict(top_p=0.5), dict(top_p=0.9), dict(min_p=0.5),
                       dict(temperature=1e-40), dict(temperature=0.0)):
                got, prob = pk.apex4_sample(dev(x), torch.tensor([u], device="cuda"), **kw)
                want, share, near = plain(x[0], F32(u), F32(kw.get("temperature", 1.0)), kw.get("top_k", 0), F32(kw.get("top_p", 1)), F32(kw.get("min_p", 0)))
                assert int(got) == want or near < V * 2.0 ** -45, (other, u, kw)
                assert float(prob) == pytest.approx(share, rel=1e-6)


def test_largest_logit(pk):
    """Settings that leave one: the lowest index of equal ones, whatever u is."""
    g = np.random.default_rng(4)
    for V in (1, 9, 5000, 70000):
        x = logits(g, 8, V, np.float16)
        x[:, V // 2] = x[:, V - 1] = 60.0
        x[5] = -0.0
        x[5, V // 3] = 0.0
        want = [V // 2] * 8
        want[5] = 0
        for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_k=1), dict(top_p=0.0),
                   dict(top_p=-0.5), dict(min_p=1.5)):
            tokens, probs = pk.apex4_sample(dev(x), dev(g.random(8).astype(F32)), **kw)
            assert tokens.tolist() == want and probs.tolist() == [1.0] * 8, kw


def test_masked_rows(pk):
    """-inf and NaN are never chosen; nothing else gives -1."""
    import torch
    g = np.random.default_rng(5)
    for V in (40, 5001, 70000):
        x = np.full((6, V), -np.inf, F32)
        x[1] = np.nan
        x[2, V - 3] = -5.0
        x[3, ::7] = g.standard_normal(len(x[3, ::7]))
        x[3, 1::7] = np.nan
        x[4, 5], x[4, 6] = 1e30, -1e30
        x[5, :] = -3e38
        for dtype in (np.float32, np.float16):
            y = x.astype(dtype) if dtype == np.float32 else np.clip(x, -65504, 65504, where=np.isfinite(x), out=x.copy()).astype(dtype)
            for kw in (dict(), dict(k=3), dict(p=0.6), dict(t=0.0), dict(k=5, p=0.5, least=0.01)):
                check(pk, y, g.random(6), **kw)
            tokens, probs = pk.apex4_sample(dev(y), torch.rand(6, device="cuda"))
            assert tokens[:3].tolist() == [-1, -1, V - 3] and probs[:3].tolist() == [0.0, 0.0, 1.0]


def test_infinite_logits(pk):
    """They share all of the weight."""
    x = np.zeros((3, 300), F32)
    x[:, [7, 100, 299]] = np.inf
    for kw in (dict(), dict(top_k=5), dict(top_p=0.99), dict(min_p=0.5), dict(temperature=float("inf"))):
        tokens, probs = pk.apex4_sample(dev(x), dev(np.array([0.1, 0.5, 0.9], F32)), **kw)
        assert tokens.tolist() == [7, 100, 299] and np.allclose(probs.cpu().numpy(), 1 / 3, rtol=1e-6)


def test_extreme_settings(pk):
    g = np.random.default_rng(6)
    x = logits(g, 4, 3001, F32)
    for t in (1e-38, 1e-5, 0.01, 30.0, 1e5):
        check(pk, x, g.random(4), t=t)
        check(pk, x, g.random(4), t=t, p=0.9, k=1000)
    check(pk, (x * 1e37).astype(F32), g.random(4), t=1e38)   # differences past binary32's range
    check(pk, (x.astype(np.float64) * 1e38).clip(-3e38, 3e38).astype(F32), g.random(4), t=1e38, p=0.8)
    tokens, probs = pk.apex4_sample(dev(x), dev(np.array([0.0, 0.25, 0.5, 1 - 2.0 ** -24], F32)), temperature=float("inf"))
    assert tokens.tolist() == [0, 750, 1500, 3000]
    # off: NaN, numbers that keep everything
    u = dev(g.random(4).astype(F32))
    want = pk.apex4_sample(dev(x), u)[0]
    for kw in (dict(top_p=float("nan")), dict(min_p=float("nan")), dict(top_p=2.0), dict(min_p=-1.0), dict(top_k=-5), dict(top_k=3001), dict(top_k=1 << 40)):
        assert pk.apex4_sample(dev(x), u, **kw)[0].equal(want), kw


def test_random_numbers_at_the_borders(pk):
    import torch
    g = np.random.default_rng(7)
    x = logits(g, 8, 2000, np.float16)
    x[:, 0] = -np.inf
    x[:, -1] = -np.inf
    u = [0.0, -1.0, float("nan"), 1.0, 7.0, float("inf"), 1 - 2.0 ** -24, 1e-38]
    tokens, _ = pk.apex4_sample(dev(x), torch.tensor(u, device="cuda"))
    assert tokens[:6].tolist() == [1, 1, 1, 1998, 1998, 1998] and int(tokens[7]) == 1
    check(pk, x, u)


def test_many_rows(pk):
    g = np.random.default_rng(8)
    x = logits(g, 700, 301, np.float16)
    check(pk, x, g.random(700), t=(0.3 + g.random(700)).astype(F32), p=0.9)


@pytest.mark.parametrize("dtype,V", [(np.float32, 50001), (np.float16, 100003), (np.float16, 131072)])
def test_few_long_rows_and_many(pk, dtype, V):
    """Long rows that several workgroups share where they are few, and one has where they are
    many: the same bits.  Lists that hold all down to the border, its bucket, or nothing."""
    import torch
    g = np.random.default_rng(V)
    B = 70
    x = logits(g, B, V, dtype)
    x[0] = 1.0
    x[1, ::2] = -np.inf
    x[2] = np.round(x[2])
    x[3, 5] = np.inf
    x[4] = np.nan
    x[5] = -np.inf
    assert pk.apex4_sample_workspace_size(6, V, torch.float16 if dtype == np.float16 else torch.float32) > 0
    assert pk.apex4_sample_workspace_size(B, V, torch.float16 if dtype == np.float16 else torch.float32) == 0
    x, u = dev(x), dev(g.random(B).astype(F32))
    for kw in (dict(), dict(temperature=0.0), dict(top_k=30), dict(top_k=20000), dict(top_p=0.9), dict(temperature=1.5, top_p=0.99), dict(min_p=0.01),
               dict(top_k=50, top_p=0.8), dict(top_k=30000, top_p=0.95), dict(top_k=V - 1), dict(temperature=0.05, top_k=V - 1, top_p=0.5),
               dict(temperature=2.0, top_p=0.97, min_p=0.001), dict(temperature=30.0, top_p=0.5)):
        whole = pk.apex4_sample(x, u, **kw)
        for i in range(0, B, 7):
            part = pk.apex4_sample(x[i:i + 7], u[i:i + 7], **kw)
            assert part[0].equal(whole[0][i:i + 7]) and part[1].equal(whole[1][i:i + 7]), (kw, i)


def test_workspace(pk):
    """The caller's, of the size asked for; a shorter one is refused."""
    import torch
    x, u = torch.randn((3, 100000), device="cuda"), torch.rand(3, device="cuda")
    need = pk.apex4_sample_workspace_size(3, 100000, torch.float32)
    work = torch.full((need + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    for kw in (dict(top_p=0.9), dict(top_k=9, top_p=0.9), dict(), dict(temperature=0.0)):
        got = pk.apex4_sample(x, u, workspace=work[:need], **kw)
        assert got[0].equal(pk.apex4_sample(x, u, **kw)[0])
    assert (work[need:] == 0xEE).all()
    with pytest.raises(pk.Apex4Error) as e:
        pk.apex4_sample(x, u, workspace=work[:need - 16])
    assert e.value.status == -7


def test_settings_for_all_rows_or_each(pk):
    import torch
    g = np.random.default_rng(9)
    x, u = dev(logits(g, 5, 900, np.float16)), dev(g.random(5).astype(F32))
    a = pk.apex4_sample(x, u, temperature=0.8, top_k=30, top_p=0.9, min_p=0.02)
    each = [torch.full((5,), v, device="cuda", dtype=torch.int32 if v == 30 else torch.float32) for v in (0.8, 30, 0.9, 0.02)]
    b = pk.apex4_sample(x, u, *each)
    assert a[0].equal(b[0]) and a[1].equal(b[1])
    tokens, probs = torch.full((7,), 9, dtype=torch.int32, device="cuda"), torch.full((7,), 9.0, device="cuda")
    pk.apex4_sample(x, u, *each, tokens=tokens[:5], probs=probs[:5])
    assert tokens[:5].equal(a[0]) and probs[:5].equal(a[1]) and tokens[5:].tolist() == [9, 9] and probs[5:].tolist() == [9.0, 9.0]
    none = pk.apex4_sample(x[:0], u[:0])
    assert none[0].shape == (0,) and none[1].shape == (0,)


def test_captured_and_on_another_stream(pk):
    import torch
    g = np.random.default_rng(10)
    for V in (3000, 70000):
        x, u = dev(logits(g, 6, V, np.float16)), dev(g.random(6).astype(F32))
        p = torch.full((6,), 0.9, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        eager = pk.apex4_sample(x, u, top_p=p, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = pk.apex4_sample(x, u, top_p=p)
        for i in range(4):
            out[0].fill_(-7)
            graph.replay()
            want = pk.apex4_sample(x, u, top_p=p)
            assert out[0].equal(want[0]) and out[1].equal(want[1])
            if i == 0:
                assert out[0].equal(eager[0])
            u.copy_(torch.rand(6, device="cuda"))
            p.mul_(0.9)


@pytest.mark.parametrize("dtype,V", [(np.float16, 1000), (np.float16, 70001), (np.float32, 131072)])
def test_two_streams_at_once(pk, dtype, V):
    """Calls under way together have a workspace each."""
    import torch
    g = np.random.default_rng(V)
    x = [dev(logits(g, 5, V, dtype)) for _ in range(2)]
    u = [dev(g.random((20, 5)).astype(F32)) for _ in range(2)]
    kw = ({"top_p": 0.9}, {"top_k": 40, "top_p": 0.8, "min_p": 0.01})
    want = [[pk.apex4_sample(x[i], u[i][n], **kw[i]) for n in range(20)] for i in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for n in range(20):
        for i in range(2):
            got[i].append(pk.apex4_sample(x[i], u[i][n], stream=sides[i], **kw[i]))
    for s in sides:
        torch.cuda.current_stream().wait_stream(s)
    for i in range(2):
        for (a, b), (c, d) in zip(got[i], want[i]):
            assert a.equal(c) and b.equal(d)


@pytest.mark.parametrize("V", [600, 50001, 131072])
@pytest.mark.parametrize("t", [1e-45, 3e-43, 1e-40, 5e-38, 1e-36, 2e-36])
def test_borders_at_the_smallest_temperatures(pk, V, t):
    """Logits some octaves of the weight apart, and hundreds to millions of octaves down, whose
    weight is nothing, all as small as such a temperature makes them; then with a largest logit that
    has no neighbour so near."""
    g = np.random.default_rng(V)
    B = 6
    u = ((np.arange(B) + g.random(B)) / B).astype(F32)
    near, far = g.random((B, V)) * 45 * t, 10.0 ** (g.random((B, V)) * 7 + 2) * t
    x = -np.where(g.random((B, V)) < 0.3, near, far).astype(F32)
    x[:, V // 2] = x[:, V // 3] = 0.0
    x[1] += F32(30 * t)    # the largest above and below 0
    x[2] -= F32(200 * t)
    x[3, V // 5:] = -np.inf
    x[4, V // 7] = 5.0     # nothing else counts
    x[5, ::2] = -3e38
    for kw in (dict(), dict(p=0.3), dict(p=0.9), dict(k=30), dict(k=V // 4), dict(k=V // 2, p=0.95), dict(least=1e-3), dict(p=0.99, least=0.05), dict(k=20, p=0.8)):
        check(pk, x, u, t=float(F32(t)), **kw)


@pytest.mark.parametrize("V", [2, 5000, 70000])
def test_the_last_octaves_that_count(pk, V):
    """Neighbours of the largest logit whose weight is 2^-30 to 2^-45 of its own are kept, however few
    steps of binary32 that is: u from 1 on takes the last kept one."""
    for m, step in ((1e8, 8.0), (1.0, 2.0 ** -24), (-(2.0 ** 20), 2.0 ** -3)):
        for steps in (1, 2, 3, 7):
            for octaves in (30.0, 34.0, 41.7, 44.5):
                x = np.full((1, V), m - 1e6 * step, F32)
                x[0, 0], x[0, -1] = m, m - steps * step
                t = steps * step * np.log2(np.e) / octaves
                for kw in (dict(), dict(least=2e-14)):
                    check(pk, x, [1.0], t=float(F32(t)), **kw)
