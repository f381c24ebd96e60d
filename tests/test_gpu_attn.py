"""Attention over the paged cache against plain 64-bit sums: single new tokens,
packed ones, windows and first tokens, page sizes, head layouts, rows that see
nothing, and NaN in every place that must not count."""
import numpy as np
import pytest

from tests import paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def decode(pk, c, **kw):
    return pk.apex4_attn_decode(dev(c.q), dev(c.k.raw), dev(c.v.raw), dev(c.table), dev(np.array(c.lens, np.int32)), c.H, c.page,
                                **{"cache": c.cache, "window": c.window, "sinks": c.sinks, **kw})


def prefill(pk, c, **kw):
    return pk.apex4_attn_prefill(dev(c.q), dev(c.start), dev(c.k.raw), dev(c.v.raw), dev(c.table),
                                 dev(np.array(c.lens, np.int32)), c.H, c.page,
                                 **{"max_q": max(c.news), "cache": c.cache, "window": c.window, "sinks": c.sinks, **kw})


def check(y, c):
    out, tol = c.expected()
    got = y.cpu().numpy().astype(np.float64)
    assert got.shape == out.shape
    bad = ~(np.abs(got - out) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.abs(got - out) / tol)))


LENS = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,Hq,H", [(16, 8, 1), (32, 6, 2), (64, 5, 5), (128, 16, 1), (16, 34, 2), (1024, 14, 2)])
def test_decode(pk, cache, D, page, Hq, H):
    c = paged.Case(7 + page, LENS, [1 if n else 0 for n in LENS], Hq, H, D, page, cache)
    # one row a sequence, the empty one's too
    c.q = np.concatenate([c.q, np.ones((1, Hq, D), np.float16)])[[int(c.start[b]) if n else -1 for b, n in enumerate(c.lens)]]
    c.news = [1] * len(LENS)
    c.start, c.T = np.arange(len(LENS) + 1, dtype=np.int32), len(LENS)
    y = decode(pk, c)
    check(y, c)
    assert (y[1] == 0).all()


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (16, 0), (33, 4), (100, 70), (64, 1), (5000, 3), (128, 100)])
def test_decode_window(pk, cache, window, sinks):
    c = paged.Case(11, [1, 40, 129, 300, 517], [1] * 5, 8, 2, 128, 16, cache, window=window, sinks=sinks)
    check(decode(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("n,page", [(5000, 16), (9001, 64)])
def test_decode_long(pk, cache, n, page):
    """Cut into many ranges, beside a short sequence that has one."""
    c = paged.Case(13, [n, 3], [1, 1], 4, 1, 64, page, cache)
    check(decode(pk, c), c)
    check(decode(pk, c, max_len=n), c)


def test_decode_growing_scores(pk):
    """Scores that rise along the sequence: the running maximum is raised again
    and again; and ones so low that a weight of binary16 would vanish."""
    for slope in (0.4, -0.4):
        c = paged.Case(17, [700], [1], 2, 1, 64, 16, "fp16", spoil=False)
        c.q[:] = 1.0
        for t in range(700):
            x = np.full((1, 64), slope * (t - 350) / 8.0, np.float16)
            c.k.put(c.table[0, t // 16], t % 16, x)
            c.K[0][t] = x
        check(decode(pk, c), c)
        check(prefill(pk, c), c)


def test_int4_scales_far_apart(pk):
    """Values of 2^-20 and of 2^10 in one sequence: their scales span binary16's
    range, the weights do not leave it; and a cache of nothing but tiny values."""
    for big in (1024.0, 2.0 ** -14):
        c = paged.Case(19, [200], [1], 4, 1, 128, 16, "int4", spoil=False)
        g = np.random.default_rng(3)
        for t in range(200):
            x = (g.standard_normal((1, 128)) * (big if t in (90, 91) else 2.0 ** -14)).astype(np.float16)
            c.v.put(c.table[0, t // 16], t % 16, x)
            c.V[0][t] = c.v.get(c.table[0, t // 16], t % 16)
        out, tol = c.expected()
        mean = np.abs(out).max()
        for y in (decode(pk, c), prefill(pk, c)):
            # 2^-11 for the weights and for the result, as much again for the rest, of the
            # weighted mean of |v|, which one output's own size may be far below
            err = np.abs(y.cpu().numpy().astype(np.float64) - out)
            assert (err <= np.minimum(tol, 2.0 ** -9 * mean * 8 + 2.0 ** -24)).all(), (big, err.max(), mean)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("zeros", ["all", "values", "keys", "first", "last"])
def test_zero_tokens(pk, cache, zeros):
    """Keys or values of nothing but zeros (scales of zero), everywhere or beside
    ordinary ones; scores far above those of the tokens with values."""
    n = 300
    c = paged.Case(67, [n], [1], 4, 1, 128, 16, cache, spoil=False)
    c.q *= np.float16(8)  # scores of some tens
    for t in range(n):
        for plane, keep, name in ((c.k, c.K, "keys"), (c.v, c.V, "values")):
            if zeros in ("all", name) or (name == "values" and ((zeros == "first" and t < 100) or (zeros == "last" and t >= 250))):
                plane.put(c.table[0, t // 16], t % 16, np.zeros((1, 128), np.float16))
                keep[0][t] = 0
    check(decode(pk, c), c)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,Hq,H", [(16, 8, 1), (64, 6, 2), (32, 5, 5), (256, 34, 2)])
def test_prefill(pk, cache, D, page, Hq, H):
    lens, news = [1, 70, 33, 64, 129, 200], [1, 1, 33, 5, 64, 130]
    c = paged.Case(23 + page, lens, news, Hq, H, D, page, cache)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (17, 0), (64, 4), (100, 70), (5000, 3)])
def test_prefill_window(pk, cache, window, sinks):
    c = paged.Case(29, [300, 65, 2, 150], [140, 65, 1, 3], 4, 2, 128, 16, cache, window=window, sinks=sinks)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,Hq,H", [(128, 8, 2), (64, 3, 3), (128, 7, 1)])
@pytest.mark.parametrize("most,window,sinks", [(2, 0, 0), (4, 0, 0), (4, 20, 3), (9, 1, 2), (9, 100, 40)])
def test_prefill_few_rows(pk, cache, D, Hq, H, most, window, sinks):
    """Few new tokens a sequence, as many as there are and fewer, with each its
    own mask in the last tile."""
    lens = [1, 2, 31, 32, 33, 40, 129, 260, 1400]
    news = [min(n, most - i % 2) for i, n in enumerate(lens)]
    c = paged.Case(71 + most, lens, news, Hq, H, D, 16, cache, window=window, sinks=sinks)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_prefill_many_sequences(pk, cache):
    """More sequences than one wave orders by length, equal lengths among them."""
    g = np.random.default_rng(5)
    news = g.integers(0, 40, 131)
    news[::7] = 33
    lens = news + g.integers(0, 3, 131) * 16
    c = paged.Case(73, lens.tolist(), news.tolist(), 3, 1, 64, 16, cache)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_prefill_split(pk, cache):
    """Few rows and a long cache: cut along the positions, and joined."""
    c = paged.Case(31, [4100, 900], [3, 2], 8, 1, 128, 64, cache)
    assert pk.apex4_attn_prefill_workspace_size(5, 2, 3, c.width, c.width * 64, 8, 1, 128, 64) > 0
    check(prefill(pk, c), c)
    c = paged.Case(37, [4100], [2], 8, 1, 64, 16, cache, window=3000, sinks=5)
    check(prefill(pk, c), c)


def test_prefill_more_new_than_cached(pk):
    """New tokens whose position would be negative see nothing: zeros."""
    import torch
    c = paged.Case(41, [5], [5], 4, 1, 64, 16, "fp16")
    q = torch.randn((9, 4, 64), dtype=torch.float16, device="cuda")
    q[4:] = dev(c.q)
    y = pk.apex4_attn_prefill(q, dev(np.array([0, 9], np.int32)), dev(c.k.raw), dev(c.v.raw), dev(c.table),
                              dev(np.array(c.lens, np.int32)), 1, 16)
    assert (y[:4] == 0).all()
    check(y[4:], c)


def test_later_tokens_do_not_reach_earlier_ones(pk):
    """Changing a token changes no row before it, bit for bit."""
    c = paged.Case(43, [150], [150], 4, 2, 128, 16, "fp16")
    a = prefill(pk, c)
    c.k.f16[c.table[0, 100 // 16], :, 100 % 16] *= -2
    c.v.f16[c.table[0, 100 // 16], :, 100 % 16] *= 3
    b = prefill(pk, c)
    import torch
    assert torch.equal(a[:100], b[:100])
    assert not torch.equal(a[100:], b[100:])


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_strided_rows_and_repeated_calls(pk, cache):
    """q out of the wider rows of a fused projection; the same bits every time,
    with and without a workspace of the caller's."""
    import torch
    c = paged.Case(47, [600, 90], [1, 1], 8, 2, 128, 16, cache)
    wide = torch.zeros((2, 8 * 128 + 512), dtype=torch.float16, device="cuda")
    q = wide[:, 256:256 + 1024].view(2, 8, 128)
    q.copy_(dev(c.q))
    args = (dev(c.k.raw), dev(c.v.raw), dev(c.table), dev(np.array(c.lens, np.int32)))
    y = pk.apex4_attn_decode(q, *args, 2, 16, cache=cache)
    check(y, c)
    need = pk.apex4_attn_decode_workspace_size(2, c.width, c.width * 16, 8, 2, 128, 16)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((2, 8, 128), float("nan"), dtype=torch.float16, device="cuda")
    for _ in range(3):
        z = pk.apex4_attn_decode(q, *args, 2, 16, cache=cache, workspace=ws, out=out)
        assert z is out and torch.equal(z, y)
    s = dev(np.array([0, 1, 2], np.int32))
    check(pk.apex4_attn_prefill(q, s, *args, 2, 16, max_q=1, cache=cache), c)


def test_table_offsets_past_32_bits(pk):
    """Pages past 4 GiB of a plane."""
    import torch
    c = paged.Case(53, [100, 40], [1, 1], 8, 8, 128, 16, "fp16")
    pages = (5 << 30) // c.k.raw.shape[1]
    used = c.k.raw.shape[0]
    planes = []
    for raw in (c.k.raw, c.v.raw):
        p = torch.zeros((pages, raw.shape[1]), dtype=torch.uint8, device="cuda")
        p[pages - used:] = dev(raw)
        planes.append(p)
    table = dev(np.where(c.table >= 0, c.table + pages - used, c.table).astype(np.int32))
    lens = dev(np.array(c.lens, np.int32))
    check(pk.apex4_attn_decode(dev(c.q), *planes, table, lens, 8, 16), c)
    check(pk.apex4_attn_prefill(dev(c.q), dev(c.start), *planes, table, lens, 8, 16, max_q=1), c)
    k = torch.randn((2, 8, 128), dtype=torch.float16, device="cuda")
    pk.apex4_kv_append(k, -k, *planes, table, lens, 16)
    a, b = pk.apex4_kv_gather(*planes, table, lens, 2, 8, 128, 16)
    assert torch.equal(a, k) and torch.equal(b, -k)


def test_ids_and_lengths_out_of_range_stay_in_bounds(pk):
    """Page ids outside the pool and lengths past the table are never addresses:
    sequences beside them are right."""
    import torch
    c = paged.Case(59, [100, 40, 20], [1, 1, 1], 4, 2, 64, 16, "fp16")
    t = c.table.copy()
    t[1] = [1 << 30, -5, c.k.raw.shape[0]] + [-1] * (c.width - 3)
    lens = np.array([100, 1 << 29, 20], np.int32)
    args = (dev(c.k.raw), dev(c.v.raw), dev(t), dev(lens))
    want, tol = c.expected()
    for y in (pk.apex4_attn_decode(dev(c.q), *args, 2, 16),
              pk.apex4_attn_prefill(dev(c.q), dev(c.start), *args, 2, 16, max_q=1)):
        got = y.cpu().numpy().astype(np.float64)
        for b in (0, 2):
            assert (np.abs(got[b] - want[b]) <= tol[b]).all()
    k = torch.ones((3, 2, 64), dtype=torch.float16, device="cuda")
    kp = args[0].clone()
    pk.apex4_kv_append(k, k, kp, args[1].clone(), args[2], args[3], 16)
    a, _ = pk.apex4_kv_gather(kp, kp, args[2], args[3], 3, 2, 64, 16)
    assert (a[0] == 1).all() and (a[1] == 0).all() and (a[2] == 1).all()


def test_side_stream_and_graph(pk):
    """On a stream of its own, and replayed from a captured graph with other
    inputs between the replays."""
    import torch
    c = paged.Case(61, [900, 31], [1, 1], 8, 2, 128, 16, "fp16")
    q, kp, vp, table = dev(c.q), dev(c.k.raw), dev(c.v.raw), dev(c.table)
    lens = dev(np.array(c.lens, np.int32))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = pk.apex4_attn_decode(q, kp, vp, table, lens, 2, 16, stream=s)
    s.synchronize()
    check(y, c)
    with torch.cuda.stream(s):
        pk.apex4_attn_decode(q, kp, vp, table, lens, 2, 16)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pk.apex4_attn_decode(q, kp, vp, table, lens, 2, 16)
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)).to(torch.float16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pk.apex4_attn_decode(q, kp, vp, table, lens, 2, 16))


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_memory_made_for_another_stream(pk, cache):
    """Output and workspace of a call on a stream that is not the current one: what
    the current stream still does to freed memory does not reach them."""
    import torch
    c = paged.Case(67, [3000, 2100], [1, 1], 8, 2, 128, 16, cache)
    q, kp, vp, table = dev(c.q), dev(c.k.raw), dev(c.v.raw), dev(c.table)
    lens = dev(np.array(c.lens, np.int32))
    need = pk.apex4_attn_decode_workspace_size(2, table.shape[1], c.width * 16, 8, 2, 128, 16)
    assert need > 0
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (q.numel() * 2, need)]
    torch.cuda._sleep(20_000_000)
    for x in freed:
        x.fill_(255)  # NaN as binary16 and as float
    del freed, x
    y = pk.apex4_attn_decode(q, kp, vp, table, lens, 2, 16, cache=cache, stream=s)
    torch.cuda.synchronize()
    check(y, c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_large_magnitude(pk, cache, D):
    """Scores of either sign of up to some 10^7, far past what an exponential holds."""
    c = paged.Case(71, [1, 2, 40, 130, 700], [1] * 5, 8, 2, D, 16, cache, sd=3000.0)
    c.q = (c.q * np.float16(2600.0)).astype(np.float16)
    s = np.concatenate([(np.abs(np.einsum("hd,thd->ht", c.q[b].astype(np.float64), np.repeat(k, 4, axis=1))) * c.scale).ravel()
                        for b, k in enumerate(c.K)])
    assert 1e7 < s.max() < 2.0 ** 26
    check(decode(pk, c), c)
    check(prefill(pk, c), c)
    n = paged.Case(73, [130, 700], [70, 33], 8, 2, D, 16, cache, sd=3000.0)
    n.q = (n.q * np.float16(2600.0)).astype(np.float16)
    check(prefill(pk, n), n)


@pytest.mark.parametrize("page,window,sinks", [(16, 0, 0), (64, 0, 0), (16, 800, 5), (128, 790, 0)])
def test_prefill_of_many_workgroups(pk, page, window, sinks):
    """The form with 256 rows a workgroup: 64 sequences x 8 key heads x 2 tiles of
    rows, and more than 12 tiles of positions."""
    lens = [1100, 900, 64, 1] + [3 + 7 * i % 60 for i in range(60)]
    news = [40, 33, 64, 1] + [1 + i % 2 for i in range(60)]
    c = paged.Case(83 + page, lens, news, 64, 8, 128, page, "fp16", window=window, sinks=sinks)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_many_rows_in_parts(pk, cache, D):
    """The join that puts several rows in a workgroup: 40 sequences of 64 heads, their
    length in several parts, most of which most sequences do not have."""
    lens = [1700, 1400, 700, 0] + [1 + 11 * i % 90 for i in range(36)]
    c = paged.Case(89 + D, lens, [1 if n else 0 for n in lens], 64, 8, D, 16, cache)
    c.q = np.concatenate([c.q, np.ones((1, 64, D), np.float16)])[[int(c.start[b]) if n else -1 for b, n in enumerate(lens)]]
    c.news = [1] * len(lens)
    c.start, c.T = np.arange(len(lens) + 1, dtype=np.int32), len(lens)
    assert pk.apex4_attn_decode_workspace_size(len(lens), c.width, c.width * 16, 64, 8, D, 16) > 0
    y = decode(pk, c)
    check(y, c)
    assert (y[3] == 0).all()
