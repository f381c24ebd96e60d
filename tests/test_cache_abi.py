"""Refusals of the paged cache's entry points (no GPU needed, nothing launched):
the documented status codes in the documented order, and the binding's own
checks."""
import ctypes

import numpy as np
import pytest

NULL = None


@pytest.fixture(scope="module")
def L():
    import os

    import paper_2606_08761_amd as pk
    if not os.path.exists(pk.LIB_PATH):
        from paper_2606_08761_amd import build
        build.build()
    return pk.lib()


BUF = np.zeros(4096, np.uint8)
P = (BUF.ctypes.data + 15) & ~15


def args(names, defaults, **kw):
    d = {**defaults, **kw}
    return [d[n] for n in names]


GEOMETRY = dict(k_pages=P, v_pages=P, n_pages=8, table=P, width=4, kv_len=P, B=2, kv_heads=2, head_dim=128, page=16, cache=0)
APPEND = dict(k=P, k_stride=256, v=P, v_stride=256, q_start=P, T=5, stream=None, **GEOMETRY)
APPEND_ORDER = ("k k_stride v v_stride q_start T k_pages v_pages n_pages table width kv_len B kv_heads head_dim page cache "
                "stream").split()
GATHER_ORDER = "k_pages v_pages n_pages table width kv_len B kv_heads head_dim page cache q_start T k v stream".split()
ATTN = dict(q=P, q_stride=1024, q_start=P, T=5, max_q=3, max_len=64, heads=8, window=0, sinks=0, scale=0.1, out=P, workspace=P,
            workspace_bytes=1 << 20, stream=None, **GEOMETRY)
DECODE_ORDER = ("q q_stride k_pages v_pages n_pages table width kv_len B max_len heads kv_heads head_dim page cache window "
                "sinks scale out workspace workspace_bytes stream").split()
PREFILL_ORDER = ("q q_stride q_start T max_q k_pages v_pages n_pages table width kv_len B max_len heads kv_heads head_dim "
                 "page cache window sinks scale out workspace workspace_bytes stream").split()

BAD_GEOMETRY = [
    (dict(k_pages=NULL), -1), (dict(v_pages=NULL), -1), (dict(table=NULL), -1), (dict(kv_len=NULL), -1),
    (dict(cache=2), -2), (dict(cache=-1), -2), (dict(head_dim=96), -2), (dict(head_dim=0), -2), (dict(page=8), -2),
    (dict(page=24), -2), (dict(page=2048), -2), (dict(kv_heads=0), -2), (dict(n_pages=0), -2), (dict(n_pages=(1 << 30) + 1), -2),
    (dict(width=0), -2), (dict(width=(1 << 20) + 1), -2), (dict(B=-1), -2), (dict(B=(1 << 24) + 1), -2),
    (dict(k_pages=P + 8), -4), (dict(v_pages=P + 4), -4), (dict(table=P + 2), -4), (dict(kv_len=P + 1), -4),
]


@pytest.mark.parametrize("bad,rc", BAD_GEOMETRY + [
    (dict(k=NULL), -1), (dict(v=NULL), -1), (dict(T=-1), -2), (dict(k_stride=248), -2), (dict(v_stride=260), -2),
    (dict(q_start=NULL), -2),  # one token a sequence, but T != B
    (dict(k=P + 8), -4), (dict(v=P + 2), -4), (dict(q_start=P + 2), -4), (dict(T=1 << 27), -2)])
def test_append(L, bad, rc):
    assert L.apex4_kv_append(*args(APPEND_ORDER, APPEND, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_GEOMETRY + [(dict(k=NULL), -1), (dict(v=NULL), -1), (dict(T=-1), -2),
                                                   (dict(q_start=NULL), -2), (dict(k=P + 8), -4), (dict(q_start=P + 1), -4)])
def test_gather(L, bad, rc):
    assert L.apex4_kv_gather(*args(GATHER_ORDER, APPEND, **bad)) == rc


BAD_ATTN = BAD_GEOMETRY + [
    (dict(q=NULL), -1), (dict(out=NULL), -1), (dict(heads=0), -2), (dict(heads=7), -2), (dict(max_len=-1), -2),
    (dict(max_len=(1 << 30) + 1), -2), (dict(window=-1), -2), (dict(sinks=-1), -2), (dict(scale=0.0), -2), (dict(scale=-1.0), -2),
    (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(q_stride=1016), -2), (dict(q_stride=1028), -2),
    (dict(q=P + 8), -4), (dict(out=P + 4), -4), (dict(workspace=P + 8), -4)]


@pytest.mark.parametrize("bad,rc", BAD_ATTN)
def test_decode(L, bad, rc):
    assert L.apex4_attn_decode(*args(DECODE_ORDER, ATTN, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_ATTN + [(dict(q_start=NULL), -1), (dict(T=-1), -2), (dict(max_q=0), -2), (dict(max_q=-1), -2),
                                               (dict(B=0), -2), (dict(q_start=P + 2), -4), (dict(T=1 << 27), -2)])
def test_prefill(L, bad, rc):
    assert L.apex4_attn_prefill(*args(PREFILL_ORDER, ATTN, **bad)) == rc


def test_sizes(L):
    b = ctypes.c_int64(-1)
    r = ctypes.byref(b)
    assert L.apex4_kv_page_bytes(0, 8, 128, 16, None) == -1
    assert L.apex4_kv_page_bytes(2, 8, 128, 16, r) == -2 and L.apex4_kv_page_bytes(0, 8, 80, 16, r) == -2
    assert b.value == -1
    assert L.apex4_kv_page_bytes(0, 8, 128, 16, r) == 0 and b.value == 8 * 16 * 256
    assert L.apex4_kv_page_bytes(1, 3, 64, 32, r) == 0 and b.value == 3 * 32 * 34
    b.value = -1
    assert L.apex4_attn_decode_workspace_size(2, 4, 64, 8, 2, 128, 16, 0, 0, None) == -1
    assert L.apex4_attn_decode_workspace_size(2, 4, 64, 7, 2, 128, 16, 0, 0, r) == -2
    assert L.apex4_attn_prefill_workspace_size(5, 2, 3, 4, 64, 8, 2, 128, 16, -1, 0, r) == -2
    assert L.apex4_attn_prefill_workspace_size(5, 2, 3, 4, 64, 8, 2, 128, 16, 0, 0, None) == -1
    assert L.apex4_pages_workspace_size(0, 1, r) == -2 and L.apex4_pages_workspace_size(8, -1, r) == -2
    assert b.value == -1
    assert L.apex4_pages_workspace_size(8, 3, r) == 0 and b.value >= 4 * (8 + 6)


PAGES = dict(pool=P, planes=4, page_bytes=64, table=P, slots=4, width=3, kv_len=P, refs=P, n_pages=8, seqs=P, new_len=P, parents=P,
             children=P, src=P, dst=P, n=2, page=16, status=P, workspace=P, workspace_bytes=1 << 12, stream=None)
BAD_STATE = [(dict(table=NULL), -1), (dict(kv_len=NULL), -1), (dict(refs=NULL), -1), (dict(slots=0), -2), (dict(width=0), -2),
             (dict(n_pages=0), -2), (dict(n=-1), -2), (dict(n=(1 << 24) + 1), -2), (dict(table=P + 2), -4), (dict(refs=P + 1), -4),
             (dict(kv_len=P + 3), -4)]
BAD_POOL = [(dict(pool=NULL), -1), (dict(planes=0), -2), (dict(page_bytes=0), -2), (dict(page_bytes=40), -2), (dict(pool=P + 8), -4)]
BAD_WORK = [(dict(status=NULL), -1), (dict(status=P + 2), -4), (dict(workspace=P + 8), -4)]


@pytest.mark.parametrize("bad,rc", BAD_STATE + BAD_WORK + [(dict(seqs=NULL), -1), (dict(new_len=NULL), -1), (dict(page=20), -2),
                                                           (dict(seqs=P + 2), -4), (dict(new_len=P + 2), -4)])
def test_reserve(L, bad, rc):
    order = "table slots width kv_len refs n_pages seqs new_len n page status workspace workspace_bytes stream".split()
    assert L.apex4_pages_reserve(*args(order, PAGES, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_STATE + BAD_POOL + BAD_WORK + [(dict(parents=NULL), -1), (dict(children=NULL), -1),
                                                                      (dict(page=0), -2), (dict(parents=P + 2), -4)])
def test_fork(L, bad, rc):
    order = ("pool planes page_bytes table slots width kv_len refs n_pages parents children n page status workspace "
             "workspace_bytes stream").split()
    assert L.apex4_pages_fork(*args(order, PAGES, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_STATE + [(dict(seqs=NULL), -1), (dict(seqs=P + 2), -4)])
def test_free(L, bad, rc):
    assert L.apex4_pages_free(*args("table slots width kv_len refs n_pages seqs n stream".split(), PAGES, **bad)) == rc


@pytest.mark.parametrize("bad,rc", [b for b in BAD_STATE if not {"n", "kv_len"} & set(b[0])] + BAD_POOL + BAD_WORK)
def test_compact(L, bad, rc):
    order = "pool planes page_bytes table slots width refs n_pages status workspace workspace_bytes stream".split()
    assert L.apex4_pages_compact(*args(order, PAGES, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_POOL + [(dict(src=NULL), -1), (dict(dst=NULL), -1), (dict(n=-1), -2), (dict(n_pages=0), -2),
                                               (dict(src=P + 2), -4), (dict(dst=P + 1), -4)])
def test_copy(L, bad, rc):
    assert L.apex4_pages_copy(*args("pool planes page_bytes n_pages src dst n stream".split(), PAGES, **bad)) == rc


def test_binding_refuses(L):
    torch = pytest.importorskip("torch")
    import paper_2606_08761_amd as pk
    with pytest.raises(ValueError):
        pk.apex4_kv_page_bytes("fp8", 8, 128, 16)
    with pytest.raises(pk.Apex4Error):
        pk.apex4_kv_page_bytes("fp16", 8, 100, 16)
    q = torch.zeros((2, 8, 128), dtype=torch.float16)
    i = torch.zeros((2, 4), dtype=torch.int32)
    planes = [torch.zeros((8, 16 * 2 * 256), dtype=torch.uint8) for _ in range(2)]
    with pytest.raises(TypeError):  # host tensors: no CPU path
        pk.apex4_attn_decode(q, *planes, i, i[:, 0], 2, 16)
    with pytest.raises(TypeError):
        pk.apex4_kv_append(q, q, *planes, i, i[:, 0], 16)


def test_pages_past_the_offsets_are_refused(L):
    """A page's bytes fit the 32-bit offsets inside it: 2^30 at most."""
    b = ctypes.c_int64(0)
    assert L.apex4_kv_page_bytes(0, 4096, 128, 1024, ctypes.byref(b)) == 0 and b.value == 1 << 30
    assert L.apex4_kv_page_bytes(0, 4097, 128, 1024, ctypes.byref(b)) == -2
    assert L.apex4_kv_page_bytes(1, 16384, 128, 1024, ctypes.byref(b)) == -2
    assert L.apex4_kv_append(*args(APPEND_ORDER, APPEND, kv_heads=8192, page=1024, k_stride=1 << 20, v_stride=1 << 20)) == -2
