"""Prompts of enough rows a key head that the kernel for many rows attends: 4-bit
values of very different sizes, bounds that a call breaks, long flat tails, and
the forms that only few-row calls reach elsewhere."""
import numpy as np
import pytest

from tests import paged
from tests.test_gpu_attn import check, dev, prefill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def rewrite(c, b, t, k=None, v=None):
    """Token t of sequence b gets other keys or values, [H, D]."""
    for x, plane, keep in ((k, c.k, c.K), (v, c.v, c.V)):
        if x is not None:
            at = c.table[b, t // c.page], t % c.page
            plane.put(*at, np.asarray(x, np.float16))
            keep[b][t] = plane.get(*at)


def check_contributions(y, c):
    """As check(), with the term of the many tokens in proportion to what a token
    contributes, not to the largest value seen: weights times values' scales are
    rounded relative to the largest of them, 2^-25 of it at most below binary16's normal
    range, and times a code of at most 8 (2^3); a value's scale is a seventh (2^-2.8) of
    its largest entry, so 2^-24.8 of the largest weight times entry, a token."""
    got = y.cpu().numpy().astype(np.float64)
    group = c.Hq // c.H
    for b, n in enumerate(c.lens):
        for i in range(c.news[b]):
            p = n - c.news[b] + i
            t = np.array([t for t in range(p + 1) if paged.seen(p, t, c.window, c.sinks)])
            for j in range(c.Hq):
                K, V = c.K[b][t, j // group], c.V[b][t, j // group]
                s = K @ c.q[c.start[b] + i, j].astype(np.float64) * c.scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out, mean, most = w @ V, w @ np.abs(V), (w * np.abs(V).max(axis=1)).max()
                tol = 2.0 ** -10 * mean + 2.0 ** -11 * np.abs(out) + len(t) * 2.0 ** -24 * most + 2.0 ** -24
                err = np.abs(got[c.start[b] + i, j] - out)
                assert (err <= tol).all(), (b, i, j, float((err / tol).max()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 0), (70, 3)])
def test_int4_values_of_other_positions_do_not_cost_precision(pk, D, window, sinks):
    """A value of thousands among ones of some hundredths: rows that do not see it (it
    is later, or before their window), in its tile and in others, keep theirs."""
    for far in (2, 40, 130, 195):
        c = paged.Case(101 + far, [200], [200], 4, 1, D, 16, "int4", window=window, sinks=sinks, spoil=False)
        g = np.random.default_rng(far)
        for t in range(200):
            rewrite(c, 0, t, v=g.standard_normal((1, D)) * (4000.0 if t == far else 0.02))
        check_contributions(prefill(pk, c), c)


@pytest.mark.parametrize("D", [64, 128])
def test_int4_large_values_of_no_weight_do_not_cost_precision(pk, D):
    """Rows that see the large value, with a score that leaves it no weight: first
    tokens with large values, a tile's only one, one a tile."""
    for far in ([0], [100], [10, 74, 138, 199]):
        c = paged.Case(113, [200], [40], 4, 1, D, 16, "int4", spoil=False)
        g = np.random.default_rng(len(far))
        c.q = np.abs(c.q)
        for t in range(200):
            big = t in far
            rewrite(c, 0, t, k=np.full((1, D), -30.0) if big else None, v=g.standard_normal((1, D)) * (4000.0 if big else 0.02))
        check_contributions(prefill(pk, c), c)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("big", [1024.0, 2.0 ** -14])
def test_int4_scales_far_apart_in_prompts(pk, D, big):
    """Values of 2^-14 and of 2^10 in one prompt, and nothing but tiny ones."""
    c = paged.Case(127, [200], [30], 4, 1, D, 16, "int4", spoil=False)
    g = np.random.default_rng(3)
    for t in range(200):
        rewrite(c, 0, t, v=g.standard_normal((1, D)) * (big if t in (90, 91, 180) else 2.0 ** -14))
    check_contributions(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,Hq,H,lens,news,max_q,window,sinks", [
    (128, 8, 1, [300, 40], [300, 40], 100, 0, 0),    # several tiles of rows, whole
    (64, 8, 1, [300, 40], [300, 40], 33, 60, 4),
    (128, 8, 1, [2500, 700], [300, 9], 20, 0, 0),    # cut along the positions
    (64, 8, 1, [2500, 700], [300, 9], 20, 1200, 4),
    (128, 4, 2, [2500, 90], [50, 3], 4, 0, 0),       # few rows
    (64, 4, 2, [900, 90], [50, 3], 1, 100, 2),
])
def test_tokens_up_to_max_q_have_their_outputs(pk, cache, D, Hq, H, lens, news, max_q, window, sinks):
    """More new tokens than the bound says: the first max_q of each sequence are
    computed, at their own positions."""
    import torch
    c = paged.Case(157, lens, news, Hq, H, D, 16, cache, window=window, sinks=sinks)
    need = pk.apex4_attn_prefill_workspace_size(c.T, len(lens), max_q, c.width, c.width * 16, Hq, H, D, 16, window, sinks)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((c.T, Hq, D), float("nan"), dtype=torch.float16, device="cuda")
    y = prefill(pk, c, max_q=max_q, workspace=ws, out=out).cpu().numpy().astype(np.float64)
    want, tol = c.expected()
    for b, n in enumerate(news):
        rows = slice(c.start[b], c.start[b] + min(n, max_q))
        assert (np.abs(y[rows] - want[rows]) <= tol[rows]).all(), b


@pytest.mark.parametrize("cache,n", [("fp16", 40000), ("int4", 100000)])
@pytest.mark.parametrize("below", [25.02, 22.3])
def test_long_flat_tails_keep_their_share(pk, cache, n, below):
    """One token of weight 1 and n - 1 of 2^-below: alone they are next to binary16's
    smallest numbers, together they are a part in some hundreds of the result."""
    import torch
    H, group, D, page, T = 8, 8, 64, 64, 512
    pages = n // page + 1
    planes = [torch.zeros((pages, pk.apex4_kv_page_bytes(cache, H, D, page)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    k = torch.zeros((n, H, D), dtype=torch.float16, device="cuda")
    v = torch.ones((n, H, D), dtype=torch.float16, device="cuda")
    k[0, :, 0] = below * np.log(2.0)
    v[0] = -1.0
    kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
    pk.apex4_kv_append(k, v, *planes, table, kv_len, page, q_start=torch.tensor([0, n], dtype=torch.int32, device="cuda"), cache=cache)
    q = torch.zeros((T, H * group, D), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    # whole lengths: the tiles of rows fill the compute units
    y = pk.apex4_attn_prefill(q, start, *planes, table, kv_len, H, page, max_q=T, cache=cache, scale=1.0).double()
    a, b = pk.apex4_kv_gather(*planes, table, kv_len, n, H, D, page, q_start=torch.tensor([0, n], dtype=torch.int32, device="cuda"), cache=cache)
    score, first, rest = a[0, 0, 0].double(), b[0, 0, 0].double(), b[1, 0, 0].double()
    share = torch.arange(n - T, n, device="cuda", dtype=torch.float64) * torch.exp(-score)
    want = ((first + share * rest) / (1 + share))[:, None, None]
    mean = ((first.abs() + share * rest.abs()) / (1 + share))[:, None, None]
    # the weight of the first is exact; a tail's weight, all equal, may be rounded the same
    # way every time: 2^-11 of it, or, below the normal range, 2^-31 of the largest one, each;
    # 2^-11 and the sums' 32 bits for the rest
    tol = 2.0 ** -11 * want.abs() + 2.0 ** -11 * (share[:, None, None] * 2) + n * 2.0 ** -31 * 2 + 2.0 ** -14 * mean
    err = (y - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,Hq,max_q", [(64, 8, 90), (128, 8, 90), (128, 4, 2)])
def test_starts_out_of_range_are_no_rows(pk, cache, D, Hq, max_q):
    """Starts of sequences that are no row numbers (a broken q_start) read and write
    nothing there; the sequences before them have their outputs."""
    import torch
    c = paged.Case(163, [300, 200, 50, 90, 70], [40, 20, 10, 10, 10], Hq, 2, D, 16, cache)
    out = torch.full((c.T, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    big = 2 ** 31 - 1
    for rest in ([60, big, big - 3, 90], [60, -5, -2 ** 31, 90], [60, big, -1, big], [60, 2 ** 24, 2 ** 30, c.T + 1]):
        out.fill_(7.0)
        start = np.array([0, 40] + rest, np.int64).astype(np.int32)
        pk.apex4_attn_prefill(dev(c.q), dev(start), dev(c.k.raw), dev(c.v.raw), dev(c.table), dev(np.array(c.lens, np.int32)),
                              2, 16, max_q=max_q, cache=cache, out=out)
        got, (want, tol) = out.cpu().numpy().astype(np.float64), c.expected()
        n = min(max_q, 40)
        assert (np.abs(got[:n] - want[:n]) <= tol[:n]).all()
        n = min(max_q, 20)
        assert (np.abs(got[40:40 + n] - want[40:40 + n]) <= tol[40:40 + n]).all()


def one_page_each(B, Hq, H, D, page, seed):
    """B sequences of up to a page: device tensors, and (out, tolerance) in 64 bits."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    planes = [torch.randn((B, H * page * D), device="cuda", generator=g).to(torch.float16).view(torch.uint8) for _ in range(2)]
    q = torch.randn((B, Hq, D), device="cuda", generator=g).to(torch.float16)
    ids = torch.randperm(B, device="cuda", generator=g).to(torch.int32)
    lens = torch.randint(1, 17, (B,), device="cuda", generator=g).to(torch.int32)
    k, v = (p.view(torch.float16).view(B, H, page, D)[ids.long(), :, :16].double().cpu().numpy() for p in planes)
    x = np.matmul(q.double().cpu().numpy().reshape(B, H, Hq // H, D), k.swapaxes(2, 3)) / np.sqrt(D)
    seen = np.arange(16) < lens.cpu().numpy()[:, None]
    x = np.where(seen[:, None, None], x, -np.inf)
    w = np.exp(x - x.max(axis=-1, keepdims=True))
    w /= w.sum(axis=-1, keepdims=True)
    out, mean = (np.matmul(w, a).reshape(B, Hq, D) for a in (v, np.abs(v)))
    # as in paged.tolerance, with at most 16 tokens of values under 8
    return q, planes, ids, lens, out, 2.0 ** -10 * mean + 2.0 ** -11 * np.abs(out) + 16 * 2.0 ** -24 * 8 + 2.0 ** -24


def test_more_workgroups_than_one_dimension_of_a_grid_holds(pk):
    """8192 sequences and max_q no better known than as all tokens: 2^24 workgroups
    of 256 threads, nearly all without rows."""
    import torch
    q, planes, ids, lens, out, tol = one_page_each(8192, 32, 2, 64, 16, 7)
    start = torch.arange(8193, device="cuda", dtype=torch.int32)
    y = pk.apex4_attn_prefill(q, start, *planes, ids[:, None].contiguous(), lens, 2, 16)
    assert (np.abs(y.cpu().numpy().astype(np.float64) - out) <= tol).all()


def test_more_parts_than_one_dimension_of_a_grid_holds(pk):
    """As many workgroups for single tokens, whose tables could hold 2^18 positions."""
    import torch
    B, H, width = 8192, 8, 256
    q, planes, ids, lens, out, tol = one_page_each(B, H, H, 64, 1024, 11)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = ids
    y = pk.apex4_attn_decode(q, *planes, table, lens, H, 1024)
    assert (np.abs(y.cpu().numpy().astype(np.float64) - out) <= tol).all()


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("zeros", ["all", "values", "keys", "first", "last"])
def test_zero_tokens_in_prompts(pk, cache, D, zeros):
    """Keys or values of nothing but zeros (scales of zero), everywhere or beside
    ordinary ones; scores far above those of the tokens with values."""
    n = 300
    c = paged.Case(131, [n], [24], 4, 1, D, 16, cache, spoil=False)
    c.q *= np.float16(8)  # scores of some tens
    zero = np.zeros((1, D))
    for t in range(n):
        some = zeros in ("all", "values") or (zeros == "first" and t < 100) or (zeros == "last" and t >= 250)
        rewrite(c, 0, t, k=zero if zeros in ("all", "keys") else None, v=zero if some else None)
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("slope", [0.4, -0.4])
def test_growing_scores_in_prompts(pk, cache, slope):
    """Scores that rise along the sequence, so that the running maximum is raised
    again and again, or fall, so that weights vanish."""
    c = paged.Case(137, [700], [24], 4, 1, 64, 16, cache, spoil=False)
    c.q[:] = 1.0
    for t in range(700):
        rewrite(c, 0, t, k=np.full((1, 64), slope * (t - 350) / 8.0))
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,page,window,sinks", [(128, 64, 0, 0), (64, 16, 0, 0), (64, 16, 3000, 5), (128, 32, 1500, 70)])
def test_prompts_cut_along_the_positions(pk, cache, D, page, window, sinks):
    """Few tiles of rows and a long cache: parts, joined; with a window, parts that
    some of the rows do not reach."""
    c = paged.Case(139, [4100, 900], [20, 12], 8, 1, D, page, cache, window=window, sinks=sinks)
    assert pk.apex4_attn_prefill_workspace_size(c.T, 2, 20, c.width, c.width * page, 8, 1, D, page, window, sinks) > 0
    check(prefill(pk, c), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
def test_prompts_on_pages_past_32_bits(pk, cache):
    """Pages past 4 GiB of a plane."""
    import torch
    c = paged.Case(149, [100, 40], [20, 17], 32, 8, 128, 16, cache)
    size, used = c.k.raw.shape[1], c.k.raw.shape[0]
    pages = (5 << 30) // size
    planes = []
    for raw in (c.k.raw, c.v.raw):
        p = torch.zeros((pages, size), dtype=torch.uint8, device="cuda")
        p[pages - used:] = dev(raw)
        planes.append(p)
    table = dev(np.where(c.table >= 0, c.table + pages - used, c.table).astype(np.int32))
    check(pk.apex4_attn_prefill(dev(c.q), dev(c.start), *planes, table, dev(np.array(c.lens, np.int32)), 8, 16, max_q=20,
                                cache=cache), c)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("page", [16, 64])
def test_prompts_beside_ids_and_lengths_out_of_range(pk, cache, page):
    """Page ids outside the pool and lengths past the table are never addresses:
    the sequences beside them are right."""
    c = paged.Case(151, [200, 90, 140], [30, 25, 40], 8, 2, 64, page, cache)
    t = c.table.copy()
    t[1] = -1
    t[1, :2] = [1 << 30, -5]
    t[1, -1] = c.k.raw.shape[0]
    y = pk.apex4_attn_prefill(dev(c.q), dev(c.start), dev(c.k.raw), dev(c.v.raw), dev(t), dev(np.array([200, 1 << 29, 140], np.int32)),
                              2, page, max_q=40, cache=cache)
    got = y.cpu().numpy().astype(np.float64)
    want, tol = c.expected()
    for b in (0, 2):
        rows = slice(c.start[b], c.start[b + 1])
        assert (np.abs(got[rows] - want[rows]) <= tol[rows]).all()


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,Hq,lens,news,at", [
    (64, 4, [150, 90], [150, 40], 100), (128, 4, [150, 90], [150, 40], 100),  # many rows
    (64, 4, [150, 90], [4, 3], 148), (128, 4, [150, 90], [4, 3], 148),        # few
    (64, 4, [700, 90], [4, 3], 698), (128, 4, [700, 90], [4, 3], 698),
])
def test_later_tokens_leave_earlier_rows_their_bits(pk, cache, D, Hq, lens, news, at):
    """Also a token that raises the running maximum of the rows that see it."""
    import torch
    c = paged.Case(167, lens, news, Hq, 2, D, 16, cache, spoil=False)
    a = prefill(pk, c)
    first = at - (lens[0] - news[0])  # the first new token that sees it
    for k, v in ((40.0, 3.0), (-40.0, 500.0)):
        rewrite(c, 0, at, k=c.K[0][at] * k, v=c.V[0][at] * v)
        b = prefill(pk, c)
        assert torch.equal(a[:first], b[:first]) and torch.equal(a[news[0]:], b[news[0]:])
        assert not torch.equal(a[first:news[0]], b[first:news[0]])
    check(b, c)
