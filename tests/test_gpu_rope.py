"""Rotary positions against the definition in 64 and 80 bits, and the append that
turns on the way against the two calls one after the other."""
import numpy as np
import pytest

from tests import paged
from tests.test_gpu_attn import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def turned(x, positions, freq, layout, mag):
    """(values, tolerance): 64-bit sums with 80-bit turns.  The kernel's product of position
    and frequency rounds to 2^-53 of the turns; sine, cosine, two products and a sum
    round to 2^-24 each, of at most |a| + |b|: 2^-22 covers them; then half a step of
    binary16 (2^-11, 2^-25 where it is subnormal)."""
    v = x.astype(np.float64)
    n = len(freq)
    t = np.asarray(positions, np.longdouble)[:, None, None] * np.asarray(freq, np.longdouble)
    angle = (2 * np.pi * (t - np.rint(t)).astype(np.longdouble)).astype(np.float64)
    c, s = np.cos(angle) * mag, np.sin(angle) * mag
    i, j = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = v[..., i], v[..., j]
    y, slack = v.copy(), np.zeros_like(v)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    off = (2.0 ** -22 + 2 * np.pi * 2.0 ** -53 * np.abs(t.astype(np.float64))) * mag * (np.abs(a) + np.abs(b))
    slack[..., i] = slack[..., j] = off
    return y, slack + 2.0 ** -11 * (np.abs(y) + slack) + 2.0 ** -25 * (slack > 0)


def rows(g, T, H, D, gap=0):
    import torch
    wide = torch.from_numpy(g.standard_normal((T, H * D + gap)).astype(np.float16)).cuda()
    return wide[:, gap // 2 // 8 * 8:][:, :H * D].view(T, H, D)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 8, 2), (16, 72, 128, 128), (33, 3, 64, 64), (7, 5, 128, 32), (5, 2, 64, 24), (9, 3, 80, 32),
                                       (3, 7, 72, 72), (4, 3, 96, 6), (2, 3, 512, 512), (2, 2, 512, 258), (1100, 3, 256, 64), (9000, 1, 64, 16)])
def test_rope(pk, layout, T, H, D, rot):
    g = np.random.default_rng(T + D + rot)
    x = rows(g, T, H, D, gap=48)
    positions = g.integers(0, 200000, T).astype(np.int32)
    freq, mag = pk.apex4_rope_freq(rot, scaling="yarn", factor=4.0)
    y = pk.apex4_rope(x, dev(positions), freq, layout=layout, scale=mag)
    want, tol = turned(x.cpu().numpy(), positions, freq.cpu().numpy(), layout, np.float32(mag).astype(np.float64))
    assert y.shape == x.shape and y.is_contiguous()
    assert (np.abs(y.cpu().numpy().astype(np.float64) - want) <= tol).all()
    # in place, in the wider rows: the same bits, and nothing else touched
    whole = x._base.clone()
    place = whole.as_strided(x.shape, x.stride(), x.storage_offset())
    assert pk.apex4_rope(place, dev(positions), freq, layout=layout, scale=mag, out=place) is place
    assert place.equal(y)
    place.copy_(x)
    assert whole.equal(x._base)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(pk, layout):
    g = np.random.default_rng(1)
    positions = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 10 ** 9 + 7, -10 ** 6], np.int32)
    x = rows(g, 8, 4, 128)
    freq, _ = pk.apex4_rope_freq(128)
    y = pk.apex4_rope(x, dev(positions), freq, layout=layout)
    want, tol = turned(x.cpu().numpy(), positions, freq.cpu().numpy(), layout, 1.0)
    assert (np.abs(y.cpu().numpy().astype(np.float64) - want) <= tol).all()
    assert y[0].equal(x[0])  # no turn: every bit


def test_infinities_and_nan_stay_in_their_pair(pk):
    import torch
    g = np.random.default_rng(2)
    x = rows(g, 2, 2, 64)
    clean = pk.apex4_rope(x, dev(np.array([3, 4], np.int32)), pk.apex4_rope_freq(32)[0])
    x[0, 1, 5], x[1, 0, 40], x[1, 1, 17] = float("nan"), float("inf"), -float("inf")
    y = pk.apex4_rope(x, dev(np.array([3, 4], np.int32)), pk.apex4_rope_freq(32)[0])
    odd = torch.zeros_like(x, dtype=torch.bool)
    odd[0, 1, 5] = odd[0, 1, 21] = odd[1, 0, 40] = odd[1, 1, 1] = odd[1, 1, 17] = True
    assert y[~odd].equal(clean[~odd]) and not torch.isfinite(y[odd]).any()
    assert torch.isinf(y[1, 0, 40])


def test_outputs_beside_the_inputs(pk):
    """Rows whose outputs are other heads of the same buffer; what overlaps is refused."""
    import torch
    g = np.random.default_rng(4)
    whole = rows(g, 33, 12, 64)
    positions = dev(g.integers(0, 5000, 33).astype(np.int32))
    freq, _ = pk.apex4_rope_freq(64)
    want = pk.apex4_rope(whole[:, 3:6], positions, freq)
    kept = whole.clone()
    for first in (0, 6, 9):
        buffer = kept.clone()
        pk.apex4_rope(buffer[:, 3:6], positions, freq, out=buffer[:, first:first + 3])
        assert buffer[:, first:first + 3].equal(want)
        rest = [h for h in range(12) if not first <= h < first + 3]
        assert buffer[:, rest].equal(kept[:, rest])
    for first in (1, 2, 4, 5):
        with pytest.raises(pk.Apex4Error):
            pk.apex4_rope(kept[:, 3:6], positions, freq, out=kept[:, first:first + 3])
    with pytest.raises(pk.Apex4Error):  # the next token's rows
        pk.apex4_rope(kept[:32, 3:6], positions[:32], freq, out=kept[1:, 3:6])
    assert kept.equal(whole)


def test_no_tokens(pk):
    import torch
    freq, _ = pk.apex4_rope_freq(64)
    x = torch.zeros((0, 4, 64), dtype=torch.float16, device="cuda")
    assert pk.apex4_rope(x, torch.zeros(0, dtype=torch.int32, device="cuda"), freq).shape == (0, 4, 64)


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,H,Hq,page,rot", [(128, 8, 64, 16, 128), (64, 3, 3, 32, 64), (128, 1, 7, 64, 32), (64, 2, 0, 16, 12), (128, 40, 40, 16, 6),
                                             (64, 5, 10, 128, 48)])
@pytest.mark.parametrize("form", ["one", "ragged", "given"])
def test_append_rope_is_rope_then_append(pk, cache, layout, D, H, Hq, page, rot, form):
    import torch
    g = np.random.default_rng(D + H + rot)
    lens = [1, 16, 50, 33, 129]
    news = [1] * 5 if form == "one" else [1, 16, 7, 0, 65]
    c = paged.Case(3, lens, news, H, H, D, page, cache, spoil=False)
    T = c.T
    qkv = rows(g, T, Hq + 2 * H, D, gap=64)
    q, k, v = torch.split(qkv, [Hq, H, H], dim=1)
    start = None if form == "one" else dev(c.start)
    own = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)]).astype(np.int32)
    positions = own if form != "given" else (own * 7 - 100).astype(np.int32)
    freq, mag = pk.apex4_rope_freq(rot, scaling="yarn", factor=2.0)
    kw = dict(layout=layout, scale=mag)
    args = [dev(c.table), dev(np.array(lens, np.int32))]
    planes = [dev(c.k.raw), dev(c.v.raw)]
    want = [p.clone() for p in planes]
    pk.apex4_kv_append(pk.apex4_rope(k, dev(positions), freq, **kw), v.contiguous(), *want, *args, page, q_start=start, cache=cache)
    got = pk.apex4_kv_append_rope(q if Hq else None, k, v, *planes, *args, page, freq, q_start=start, cache=cache,
                                  positions=dev(positions) if form == "given" else None, **kw)
    assert all(a.equal(b) for a, b in zip(planes, want))
    if Hq:
        assert got.is_contiguous() and got.equal(pk.apex4_rope(q, dev(positions), freq, **kw))
    else:
        assert got is None


def test_tokens_without_a_place(pk):
    """Before a sequence's start, past its table, on no page, behind the last sequence:
    the cache is left alone; queries behind the last sequence too."""
    import torch
    H, D, page = 2, 64, 16
    g = np.random.default_rng(4)
    table = dev(np.array([[0, -1], [9, 2]], np.int32))   # sequence 0 has one page; page 9 is not of the pool
    lens = dev(np.array([18, 3], np.int32))
    start = dev(np.array([0, 20, 24], np.int32))          # 20 new tokens of 18; 4 of 3; 2 rows behind
    T = 26
    q, k, v = (rows(g, T, H, D) for _ in range(3))
    planes = [torch.zeros((4, H * page * D * 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    freq, _ = pk.apex4_rope_freq(D)
    out = torch.full((T, H, D), 7.0, dtype=torch.float16, device="cuda")
    pk.apex4_kv_append_rope(q, k, v, *planes, table, lens, page, freq, q_start=start, out=out)
    positions = np.concatenate((np.arange(20) - 2, np.arange(4) - 1, [0, 0])).astype(np.int32)
    assert out[:24].equal(pk.apex4_rope(q, dev(positions), freq)[:24]) and (out[24:] == 7.0).all()
    want = torch.zeros((4, H, page, D), dtype=torch.float16, device="cuda")
    want[0] = pk.apex4_rope(k, dev(positions), freq)[2:18].transpose(0, 1)
    assert planes[0].view(torch.float16).view(4, H, page, D).equal(want)
    want[0] = v[2:18].transpose(0, 1)
    assert planes[1].view(torch.float16).view(4, H, page, D).equal(want)


def test_captured_and_on_another_stream(pk):
    """Replays follow the lengths on the device; work on a side stream waits for nothing."""
    import torch
    g = np.random.default_rng(8)
    H, D, B = 8, 128, 4
    freq, _ = pk.apex4_rope_freq(D)
    q, k, v = rows(g, B, 32, D), rows(g, B, H, D), rows(g, B, H, D)
    cache = pk.PagedKVCache(1, 32, B, H, D, 16, 64)
    assert cache.reserved(cache.reserve(list(range(B)), [60] * B))
    table, _ = cache.batch(list(range(B)))
    lens = torch.tensor([1, 5, 16, 17], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = cache.append_rope(0, q, k, v, (table, lens), freq, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert eager.equal(pk.apex4_rope(q, lens - 1, freq))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.append_rope(0, q, k, v, (table, lens), freq)
        turned_q = pk.apex4_rope(q, lens, freq)
    for i in range(4):
        lens += 7
        out.fill_(0)
        graph.replay()
        assert out.equal(pk.apex4_rope(q, lens - 1, freq)) and turned_q.equal(pk.apex4_rope(q, lens, freq))
        kk, vv = cache.gather(0, B, (table, lens))
        assert kk.equal(pk.apex4_rope(k, lens - 1, freq)) and vv.equal(v)
