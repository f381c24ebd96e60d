"""The paged cache's tokens and pages: what append writes and leaves alone, what
gather reads, and the page calls against a plain model of the same state."""
import numpy as np
import pytest

from tests import paged
from tests.test_gpu_attn import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,H,page", [(128, 8, 16), (64, 3, 32), (128, 1, 64), (64, 40, 16)])
@pytest.mark.parametrize("one", [True, False])
def test_append_and_gather(pk, cache, D, H, page, one):
    import torch
    g = np.random.default_rng(D + H)
    lens = [1, 16, 50, 33, 129]
    news = [1] * 5 if one else [1, 16, 7, 0, 65]
    c = paged.Case(3, lens, news, H, H, D, page, cache, spoil=False)
    T = c.T
    wide = torch.from_numpy(g.standard_normal((T, 2 * H * D + 64)).astype(np.float16)).cuda()
    k, v = wide[:, :H * D].view(T, H, D), wide[:, H * D + 64:].view(T, H, D)
    start = None if one else dev(c.start)
    kp, vp, table, kv_len = dev(c.k.raw), dev(c.v.raw), dev(c.table), dev(np.array(lens, np.int32))
    pk.apex4_kv_append(k, v, kp, vp, table, kv_len, page, q_start=start, cache=cache)
    for x, plane in ((k, c.k), (v, c.v)):
        x = x.cpu().numpy()
        for b, n in enumerate(lens):
            for i in range(news[b]):
                t = n - news[b] + i
                plane.put(c.table[b, t // page], t % page, x[c.start[b] + i])
    # every byte: the new tokens written, all else as it was
    assert np.array_equal(kp.cpu().numpy(), c.k.raw)
    assert np.array_equal(vp.cpu().numpy(), c.v.raw)
    gk, gv = pk.apex4_kv_gather(kp, vp, table, kv_len, T, H, D, page, q_start=start, cache=cache)
    for got, plane in ((gk, c.k), (gv, c.v)):
        want = np.stack([plane.get(c.table[b, t // page], t % page) for b, n in enumerate(lens)
                         for t in range(n - news[b], n)])
        assert np.array_equal(got.cpu().numpy(), want.astype(np.float16))


def test_append_quantizes_as_the_quantizer_does(pk):
    """Codes and scales of apex4_quantize_act with G = head_dim, ties, zero rows
    and subnormal scales among them."""
    import torch
    H, D, page, T = 4, 128, 16, 64
    g = torch.Generator().manual_seed(5)
    x = torch.randn((T, H, D), generator=g).to(torch.float16)
    x[0] = 0
    x[1] *= 2.0 ** -20
    x[2] = (torch.randint(-14, 15, (H, D), generator=g) * 0.5).to(torch.float16)   # ties
    x[2, :, 0] = 7.0
    x[3] = 60000.0
    x = x.cuda()
    q, s = pk.apex4_quantize_act(x.reshape(T * H, D), D)
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    planes = [torch.zeros((4, pk.apex4_kv_page_bytes("int4", H, D, page)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    pk.apex4_kv_append(x, x, *planes, table, lens, page, q_start=torch.tensor([0, T], dtype=torch.int32, device="cuda"), cache="int4")
    n = H * page * D // 2
    for p in planes:
        codes = p[:, :n].reshape(4, H, page, D // 2).transpose(1, 2).reshape(T, H, D // 2)
        scales = p[:, n:].contiguous().view(torch.float16).reshape(4, H, page).transpose(1, 2).reshape(T, H)
        assert torch.equal(codes.reshape(T * H, -1), q)
        assert torch.equal(scales.reshape(T * H, 1), s)


def test_many_sequences_share_a_call(pk):
    """300 sequences of no, one and several new tokens."""
    import torch
    g = np.random.default_rng(9)
    news = g.integers(0, 4, 300)
    lens = news + g.integers(0, 30, 300)
    start = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
    table = g.permutation(900)[:900].reshape(300, 3).astype(np.int32)
    T, H, D = int(start[-1]), 2, 64
    k = torch.randn((T, H, D), device="cuda", dtype=torch.float16)
    kp, vp = (torch.zeros((900, 16 * H * D * 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    args = (dev(table), dev(lens.astype(np.int32)))
    pk.apex4_kv_append(k, -k, kp, vp, *args, 16, q_start=dev(start))
    a, b = pk.apex4_kv_gather(kp, vp, *args, T, H, D, 16, q_start=dev(start))
    assert torch.equal(a, k) and torch.equal(b, -k)
    full = kp.view(torch.float16).view(900, H, 16, D).cpu().numpy()
    for s in (0, 17, 150, 299):
        for i in range(news[s]):
            t = lens[s] - news[s] + i
            assert np.array_equal(full[table[s, t // 16], :, t % 16], k[start[s] + i].cpu().numpy())


class Model:
    """The page calls on the host, one at a time."""

    def __init__(self, pool, slots, width, page):
        self.pool, self.page = pool, page
        self.table = np.full((slots, width), -1, np.int32)
        self.len = np.zeros(slots, np.int32)
        self.refs = np.zeros(pool.shape[1], np.int32)

    def need(self, n):
        return -(-int(n) // self.page)

    def free_pages(self):
        return [p for p in range(len(self.refs)) if self.refs[p] == 0]

    def reserve(self, seqs, new_len):
        if any(self.need(n) > self.table.shape[1] for n in new_len):
            return -1
        want = [max(self.need(n) - self.need(self.len[s]), 0) for s, n in zip(seqs, new_len)]
        free = self.free_pages()
        if sum(want) > len(free):
            return 1
        for s, n, w in zip(seqs, new_len, want):
            have = self.need(self.len[s])
            for i in range(w):
                p = free.pop(0)
                self.table[s, have + i] = p
                self.refs[p] = 1
            self.len[s] = max(self.len[s], n)
        return 0

    def fork(self, parents, children):
        part = [self.len[p] % self.page != 0 for p in parents]
        free = self.free_pages()
        if sum(part) > len(free):
            return sum(part) - len(free)
        for p, c, x in zip(parents, children, part):
            full = self.len[p] // self.page
            self.table[c] = -1
            self.table[c, :full] = self.table[p, :full]
            for i in self.table[c, :full]:
                self.refs[i] += 1
            if x:
                new = free.pop(0)
                self.table[c, full] = new
                self.refs[new] = 1
                self.pool[:, new] = self.pool[:, self.table[p, full]]
            self.len[c] = self.len[p]
        return 0

    def free(self, seqs):
        for s in seqs:
            for i in self.table[s]:
                if i >= 0:
                    self.refs[i] -= 1
            self.table[s] = -1
            self.len[s] = 0

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        src = [p for p in live if p >= len(live)]
        dst = [p for p in range(len(live)) if self.refs[p] == 0]
        to = {p: p for p in live} | dict(zip(src, dst))
        for a, b in zip(src, dst):
            self.pool[:, b] = self.pool[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = np.vectorize(lambda i: to[i] if i >= 0 else -1, otypes=[np.int32])(self.table)
        return len(live)


@pytest.mark.parametrize("pages,slots,width,page,size,steps", [
    (40, 12, 6, 16, 48, 60),          # runs out of pages often
    (300, 20, 9, 32, 16 * 1027, 60),  # page data that ends inside a 16 KB piece
    (9000, 2100, 5, 16, 16, 30),      # more slots than a workgroup takes at a time
    (16384, 2100, 5, 16, 16, 30),     # as many pages as it does
    (40001, 2100, 30, 16, 16, 30),    # and more
])
def test_page_calls(pk, pages, slots, width, page, size, steps):
    import torch
    g = np.random.default_rng(pages)
    pool = g.integers(0, 256, (3, pages, size), dtype=np.uint8)
    m = Model(pool.copy(), slots, width, page)
    d_pool, table, kv_len, refs = dev(pool), dev(m.table), dev(m.len), dev(m.refs)
    outcomes = set()
    for step in range(steps):
        used, empty = np.flatnonzero(m.len > 0), np.flatnonzero(m.len == 0)
        kind = g.choice(["reserve", "reserve", "fork", "free", "compact"])
        most = 3 if slots < 100 else 1500
        if kind == "reserve":
            seqs = g.permutation(slots)[:g.integers(1, most + 3)].astype(np.int32)
            new = np.maximum(m.len[seqs], 0) + g.integers(0, 2 * page, len(seqs)) * (g.random(len(seqs)) < 0.8)
            new = np.minimum(new, width * page + (1 if g.random() < 0.1 else 0)).astype(np.int32)
            want = m.reserve(seqs, new)
            got = int(pk.apex4_pages_reserve(table, kv_len, refs, dev(seqs), dev(new), page).item())
            assert (got > 0) == (want > 0) and (got == want or want > 0)
            outcomes.add((kind, np.sign(want)))
        elif kind == "fork" and len(used) and len(empty):
            n = min(len(empty), int(g.integers(1, most + 1)))
            par = g.choice(used, n).astype(np.int32)
            ch = g.permutation(empty)[:n].astype(np.int32)
            want = m.fork(par, ch)
            assert int(pk.apex4_pages_fork(d_pool, table, kv_len, refs, dev(par), dev(ch), page).item()) == want
            outcomes.add((kind, np.sign(want)))
        elif kind == "free" and len(used):
            seqs = g.permutation(used)[:g.integers(1, most + 1)].astype(np.int32)
            m.free(seqs)
            pk.apex4_pages_free(table, kv_len, refs, dev(np.append(seqs, np.int32(slots + 5))))
        else:
            assert int(pk.apex4_pages_compact(d_pool, table, refs).item()) == m.compact()
        assert np.array_equal(table.cpu().numpy(), m.table), (step, kind)
        assert np.array_equal(kv_len.cpu().numpy(), m.len), (step, kind)
        assert np.array_equal(refs.cpu().numpy(), m.refs), (step, kind)
        live = m.refs > 0  # a page's data counts while it is held
        assert np.array_equal(d_pool.cpu().numpy()[:, live], m.pool[:, live]), (step, kind)
    assert ("reserve", 0) in outcomes and ("fork", 0) in outcomes
    if pages == 40:
        assert ("reserve", 1) in outcomes


@pytest.mark.parametrize("pages", [1, 15, 16, 17, 16384, 16385, 50000])
@pytest.mark.parametrize("held", ["none", "all", "low", "high", "mixed"])
def test_compact(pk, pages, held):
    """Nothing to move, everything to move, and pools that end at a boundary."""
    import torch
    g = np.random.default_rng(pages)
    refs = {"none": np.zeros(pages), "all": np.ones(pages), "low": np.arange(pages) < pages // 3, "high": np.arange(pages) >= pages - pages // 3,
            "mixed": g.integers(0, 3, pages)}[held].astype(np.int32)
    live = np.flatnonzero(refs)
    m = Model(np.arange(pages, dtype=np.uint8).repeat(16).reshape(1, pages, 16).copy(), max(1, len(live)), 1, 16)
    m.pool[0, :, :8] = np.arange(pages, dtype=np.int64).view(np.uint8).reshape(pages, 8)
    m.refs, m.table = refs, (live[:, None] if len(live) else np.full((1, 1), -1)).astype(np.int32)
    pool, table, d_refs = dev(m.pool), dev(m.table), dev(refs)
    assert int(pk.apex4_pages_compact(pool, table, d_refs).item()) == m.compact() == len(live)
    assert np.array_equal(table.cpu().numpy(), m.table) and np.array_equal(d_refs.cpu().numpy(), m.refs)
    assert np.array_equal(pool.cpu().numpy()[:, :len(live)], m.pool[:, :len(live)])


def test_copy_pages(pk):
    import torch
    pool = torch.randint(0, 256, (4, 50, 16 * 2051), dtype=torch.uint8, device="cuda")
    want = pool.clone()
    src, dst = [3, 9, 9, 60, 4, -1], [20, 21, 49, 22, 99, 23]
    for s, d in zip(src, dst):
        if 0 <= s < 50 and 0 <= d < 50:
            want[:, d] = want[:, s]
    ids = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst)]
    pk.apex4_pages_copy(pool, *ids)
    assert torch.equal(pool, want)


def test_a_sequences_life(pk):
    """Reserve, append, fork, append, compact and free through PagedKVCache: what
    a sequence holds stays its own."""
    import torch
    for kind in ("fp16", "int4"):
        c = pk.PagedKVCache(layers=2, pages=64, slots=6, kv_heads=2, head_dim=64, page=16, max_len=200, cache=kind)
        held = {}
        g = torch.Generator(device="cuda").manual_seed(1)

        def grow(s, n):
            new = torch.randn((2, n, 2, 64), device="cuda", generator=g).to(torch.float16)
            total = len(held.get(s, [[], []])[0]) + n
            assert c.reserved(c.reserve([s], [total]))
            start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            for layer in range(2):
                c.append(layer, new[layer], -new[layer], c.batch([s]), start)
            old = held.get(s, [new[0][:0], new[1][:0]])
            held[s] = [torch.cat((old[i], new[i])) for i in range(2)]

        def look():
            for s, x in held.items():
                n = len(x[0])
                start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
                for layer in range(2):
                    k, v = c.gather(layer, n, c.batch([s]), start)
                    want = x[layer]
                    if kind == "fp16":
                        assert torch.equal(k, want) and torch.equal(v, -want)
                    else:
                        # half a step of the scale amax / 7, and its rounding to binary16
                        step = want.float().abs().amax(dim=-1, keepdim=True) / 7 * (1 + 2 ** -9)
                        assert ((k.float() - want.float()).abs() <= 0.51 * step).all()

        grow(0, 50)
        grow(3, 16)
        assert c.reserved(c.fork([0, 0, 3], [1, 2, 4]))
        held[1], held[2], held[4] = list(held[0]), list(held[0]), list(held[3])
        for s, n in ((1, 30), (0, 3), (2, 1), (4, 17)):
            grow(s, n)
            look()
        c.free([0])
        del held[0]
        live = int(c.compact().item())
        assert live == len(set(c.table[c.table >= 0].tolist())) and int(c.table.max()) == live - 1
        look()
        c.free([1, 2, 3, 4])
        assert int(c.refs.abs().sum()) == 0 and int(c.kv_len.sum()) == 0


def test_an_empty_status_is_refused(pk):
    import torch
    c = pk.PagedKVCache(layers=1, pages=4, slots=2, kv_heads=1, head_dim=64)
    none = torch.empty((0,), dtype=torch.int32, device="cuda")
    for call in (lambda: c.reserve([0], [5], status=none), lambda: c.fork([0], [1], status=none), lambda: c.compact(status=none)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("cache", ["fp16", "int4"])
@pytest.mark.parametrize("D,H", [(64, 3), (128, 2)])
def test_append_of_long_prompts(pk, cache, D, H):
    """Enough tokens that a workgroup takes several, of more than one sequence: the
    same bytes as token after token."""
    import torch
    lens = [3500, 1, 2, 1999, 0, 530, 3]
    page, T = 32, sum(lens)
    rows = [-(-n // page) for n in lens]
    order = torch.randperm(sum(rows) + 2, generator=torch.Generator().manual_seed(D))
    table = torch.full((len(lens), max(rows)), -1, dtype=torch.int32)
    for b, n in enumerate(rows):
        table[b, :n] = order[sum(rows[:b]):sum(rows[:b]) + n]
    start = torch.tensor([sum(lens[:b]) for b in range(len(lens) + 1)], dtype=torch.int32).cuda()
    table, kv_len = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    g = torch.Generator(device="cuda").manual_seed(D + 1)
    k, v = (torch.randn((T, H, D), device="cuda", generator=g).to(torch.float16) for _ in range(2))
    size = pk.apex4_kv_page_bytes(cache, H, D, page)
    kp, vp, kq, vq = (torch.zeros((sum(rows) + 2, size), dtype=torch.uint8, device="cuda") for _ in range(4))
    pk.apex4_kv_append(k, v, kp, vp, table, kv_len, page, q_start=start, cache=cache)
    # one token at a time to each of up to 512 "sequences", which share their tables
    at = torch.cat([torch.stack([torch.full((n,), b), torch.arange(1, n + 1)]) for b, n in enumerate(lens) if n], 1).cuda()
    for i in range(0, T, 512):
        b, n = at[0, i:i + 512], at[1, i:i + 512].to(torch.int32)
        pk.apex4_kv_append(k[i:i + 512], v[i:i + 512], kq, vq, table[b].contiguous(), n, page, cache=cache)
    assert torch.equal(kp, kq) and torch.equal(vp, vq) and bool(kp.any())
    gk, gv = pk.apex4_kv_gather(kp, vp, table, kv_len, T, H, D, page, q_start=start, cache=cache)
    for i in range(0, T, 512):
        b, n = at[0, i:i + 512], at[1, i:i + 512].to(torch.int32)
        a, c = pk.apex4_kv_gather(kp, vp, table[b].contiguous(), n, len(n), H, D, page, cache=cache)
        assert torch.equal(a, gk[i:i + 512]) and torch.equal(c, gv[i:i + 512])
    if cache == "fp16":
        assert torch.equal(gk, k) and torch.equal(gv, v)
