"""PagedKVCache and the page calls where a call's bounds meet: lengths past max_len
that the table still holds, more pages asked for than there are, lists on other
streams."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def test_lists_belong_to_the_stream_of_the_call(pk, monkeypatch):
    """The memory of a list's tensor goes to no call on another stream: the current
    one's next small tensors are not made of it."""
    import torch

    from paper_2606_08761_amd import cache
    c = pk.PagedKVCache(layers=1, pages=64, slots=16, kv_heads=1, head_dim=64, page=16, max_len=64)
    made = []

    def watched(name, at):
        call = getattr(cache, name)

        def run(*args, **kw):
            made.extend(args[i].data_ptr() for i in at)
            return call(*args, **kw)
        monkeypatch.setattr(cache, name, run)

    watched("apex4_pages_reserve", (3, 4))
    watched("apex4_pages_fork", (4, 5))
    watched("apex4_pages_free", (3,))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    others = []

    def then():
        torch.cuda._sleep(200_000)
        others.extend(torch.full((1,), 7, dtype=torch.int32, device="cuda") for _ in range(8))
        assert not set(made) & {x.data_ptr() for x in others}

    for i in range(6):
        status = c.reserve([i], [20 + i], stream=s)
        then()
        s.synchronize()
        assert c.reserved(status)
    for i in range(6):
        status = c.fork([i], [6 + i], stream=s)
        then()
        s.synchronize()
        assert c.reserved(status)
    assert c.kv_len.tolist() == [*range(20, 26), *range(20, 26), 0, 0, 0, 0]
    for i in range(0, 12, 2):
        c.free([i], stream=s)
        then()
    s.synchronize()
    assert c.kv_len.tolist() == [0 if i % 2 == 0 else 20 + i % 6 for i in range(12)] + [0] * 4
    assert len(made) == 6 * 2 + 6 * 2 + 6


@pytest.mark.parametrize("kind", ["fp16", "int4"])
def test_lengths_up_to_the_tables_end_are_seen(pk, kind):
    """max_len inside a page: what reserve gives, attention sees."""
    import torch
    c = pk.PagedKVCache(layers=1, pages=8, slots=2, kv_heads=2, head_dim=64, page=16, max_len=20, cache=kind)
    g = torch.Generator(device="cuda").manual_seed(2)
    n = 30
    assert c.reserved(c.reserve([1], [n]))
    assert not c.reserved(c.reserve([0], [33]))  # does not fit the table
    k, v = (torch.randn((n, 2, 64), device="cuda", generator=g).to(torch.float16) for _ in range(2))
    q = torch.randn((n, 4, 64), device="cuda", generator=g).to(torch.float16)
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    b = c.batch([1])
    c.append(0, k, v, b, start)
    args = (*c.planes[0], *b, 2, 16)
    assert torch.equal(c.decode(0, q[-1:], b), pk.apex4_attn_decode(q[-1:], *args, cache=kind))
    assert torch.equal(c.prefill(0, q, b, start, n), pk.apex4_attn_prefill(q, start, *args, max_q=n, cache=kind))
    assert torch.equal(c.prefill(0, q[-2:], b, torch.tensor([0, 2], dtype=torch.int32, device="cuda"), 2),
                       pk.apex4_attn_prefill(q[-2:], torch.tensor([0, 2], dtype=torch.int32, device="cuda"), *args, max_q=2, cache=kind))


@pytest.mark.parametrize("pages,children", [(4, 6), (4, 3), (4, 4), (3, 2000)])
def test_fork_counts_the_pages_that_are_missing(pk, pages, children):
    """Also where the children outnumber the pool's pages."""
    import torch
    c = pk.PagedKVCache(layers=1, pages=pages, slots=children + 1, kv_heads=1, head_dim=64, page=16, max_len=64)
    assert c.reserved(c.reserve([0], [5]))
    before = [x.clone() for x in (c.table, c.kv_len, c.refs)]
    missing = max(0, children - (pages - 1))
    assert int(c.fork([0] * children, list(range(1, children + 1))).item()) == missing
    if missing:  # nothing has changed
        assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.kv_len, c.refs)))
