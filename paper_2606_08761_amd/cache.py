"""Paged key-value cache and the attention that reads it: bindings of the
``apex4_kv_*``, ``apex4_attn_*`` and ``apex4_pages_*`` calls of include/apex4.h,
and ``PagedKVCache``, which keeps their tensors.

A plane (the keys or the values of one layer) is uint8 [pages, page bytes];
``cache`` is "fp16" or "int4" (SymQuant codes, one scale for a token's head).
Table, lengths and sequence numbers are int32 tensors on the device.

    c = PagedKVCache(layers=2, pages=512, slots=8, kv_heads=8, max_len=2048)
    c.reserve(seqs, new_len)                      # pages for what comes
    b = c.batch(seqs)                             # their rows of the table, their lengths
    c.append(layer, k, v, b, q_start)             # the new tokens' keys and values
    q = c.append_rope(layer, q, k, v, b, freq, q_start)  # or: with rotary positions, q's too
    y = c.prefill(layer, q, b, q_start, max_q)    # a prompt's attention
    y = c.decode(layer, q, b)                     # one new token a sequence
"""
from __future__ import annotations

import ctypes
import functools
import math

from . import Apex4Error, _check, _dev, _stream, _torch, lib

KV_CACHES = {"fp16": 0, "int4": 1}
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}


def _kind(cache):
    try:
        return KV_CACHES[cache]
    except KeyError:
        raise ValueError("cache must be 'fp16' or 'int4'") from None


def _layout(layout):
    try:
        return ROPE_LAYOUTS[layout]
    except KeyError:
        raise ValueError("layout must be 'half' or 'interleaved'") from None


def _one_device(t, *others):
    """The tensors of a call (or None) lie on the current device, where it launches."""
    i = t.get_device()
    for o in others:
        if o is not None and o.get_device() != i:
            raise ValueError("all tensors of a call must be on one device")
    if i != _torch()._C._cuda_getDevice():  # 0.1 us; torch.cuda.current_device() takes 0.4
        raise ValueError("the tensors of a call must be on the current device")


def _ptr(t, dtype, name):
    """_dev, quicker where nothing is wrong (small calls are bound by this)."""
    try:
        if t.dtype is dtype and t.is_cuda and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _dev(t, dtype, name)


def _index(t, name):
    return _ptr(t, _torch().int32, name)


def _rows(t, name):
    """Pointer and row stride of [T, heads, D] float16 whose heads are contiguous."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype is not torch.float16:
        raise TypeError(f"{name} must be {torch.float16}, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    T, H, D = t.shape
    row, head, one = t.stride()
    if (one != 1 and D > 1) or (head != D and H > 1):
        raise ValueError(f"the heads of {name}'s rows must be contiguous")
    return t.data_ptr(), row if T > 1 else H * D


def _freq(freq):
    """Pointer of freq [rot / 2], and rot."""
    p = _ptr(freq, _torch().float64, "freq")
    if freq.dim() != 1:
        raise ValueError("freq must be [rot / 2]")
    return p, 2 * freq.shape[0]


def _planes(k_pages, v_pages, kv_heads, head_dim, page, cache):
    torch = _torch()
    kp, vp = _ptr(k_pages, torch.uint8, "k_pages"), _ptr(v_pages, torch.uint8, "v_pages")
    n = apex4_kv_page_bytes(cache, kv_heads, head_dim, page)
    shape = k_pages.shape
    if len(shape) != 2 or shape[1] != n or v_pages.shape != shape:
        raise ValueError(f"k_pages and v_pages must be [pages, {n}]: {kv_heads} heads of {head_dim}, {page} tokens a page, "
                         f"{cache}")
    return kp, vp, shape[0]


def _tables(table, kv_len):
    shape = table.shape
    if len(shape) != 2 or kv_len.shape != shape[:1]:
        raise ValueError("table must be [B, width] and kv_len [B]")
    i32 = _torch().int32
    return _ptr(table, i32, "table"), shape[1], _ptr(kv_len, i32, "kv_len"), shape[0]


def _starts(q_start, B):
    if q_start is None:
        return None
    if q_start.dim() != 1 or q_start.shape[0] != B + 1:
        raise ValueError("q_start must be [B + 1]")
    return _index(q_start, "q_start")


def _empty(like, shape, dtype, stream):
    """Memory of the stream that the call runs on: what an earlier owner on another
    stream still has under way does not reach it, nor this call its next owner."""
    if stream is None:
        return like.new_empty(shape) if like.dtype is dtype else like.new_empty(shape, dtype=dtype)
    with _torch().cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _output(out, shape, like, stream):
    if out is None:
        return _empty(like, shape, _torch().float16, stream)
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"the output must be {tuple(shape)}")
    return out


def _output_like(out, q, stream):
    """_output of q's shape; quicker where q has no gaps."""
    if out is None and stream is None and q.is_contiguous():
        return _torch().empty_like(q)
    return _output(out, q.shape, q, stream)


def _workspace(workspace, need, like, stream):
    """(pointer, bytes): the caller's, or one made here where one is needed."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = _empty(like, (need,), _torch().uint8, stream)
        return workspace.data_ptr(), need, workspace
    return _dev(workspace, _torch().uint8, "workspace"), workspace.numel(), workspace


@functools.lru_cache(maxsize=256)
def apex4_kv_page_bytes(cache: str, kv_heads: int, head_dim: int, page: int) -> int:
    """Bytes of a page of one plane."""
    b = ctypes.c_int64(0)
    _check("apex4_kv_page_bytes", lib().apex4_kv_page_bytes(_kind(cache), kv_heads, head_dim, page, ctypes.byref(b)))
    return int(b.value)


def apex4_kv_append(k, v, k_pages, v_pages, table, kv_len, page: int, q_start=None, cache: str = "fp16", stream=None):
    """New tokens' keys and values, [T, kv_heads, head_dim] float16 with any row
    stride that is a multiple of 8, into the cache.  q_start None: one a sequence."""
    (T, H, D) = k.shape
    if v.shape != k.shape:
        raise ValueError("k and v must have one shape")
    kp, ks = _rows(k, "k")
    vp, vs = _rows(v, "v")
    kpp, vpp, n = _planes(k_pages, v_pages, H, D, page, cache)
    tp, width, lp, B = _tables(table, kv_len)
    rc = lib().apex4_kv_append(kp, ks, vp, vs, _starts(q_start, B), T, kpp, vpp, n, tp, width, lp, B, H, D, page,
                               _kind(cache), _stream(k, stream))
    _check("apex4_kv_append", rc)


def apex4_kv_append_rope(q, k, v, k_pages, v_pages, table, kv_len, page: int, freq, layout: str = "half", scale: float = 1.0,
                         q_start=None, positions=None, cache: str = "fp16", out=None, stream=None):
    """apex4_kv_append with the keys turned by their positions (None: their places in
    the sequences), freq and scale as apex4_rope.  q [T, heads, head_dim] (or None) is
    turned too, into ``out`` [T, heads, head_dim] (made here when None), which is returned."""
    torch = _torch()
    (T, H, D) = k.shape
    if v.shape != k.shape:
        raise ValueError("k and v must have one shape")
    kp, ks = _rows(k, "k")
    vp, vs = _rows(v, "v")
    fp, rot = _freq(freq)
    qp, qs, heads, op = None, 0, 0, None
    given = out
    if q is not None:
        qp, qs = _rows(q, "q")
        rows, heads, size = q.shape
        if rows != T or size != D:
            raise ValueError("q must be [T, heads, head_dim], as k")
        if out is None:
            out = _empty(q, (T, heads, D), torch.float16, stream)
            op = out.data_ptr()
        else:
            op = _ptr(_output(out, (T, heads, D), q, stream), torch.float16, "out")
    if positions is not None and tuple(positions.shape) != (T,):
        raise ValueError("positions must be [T]")
    kpp, vpp, n = _planes(k_pages, v_pages, H, D, page, cache)
    tp, width, lp, B = _tables(table, kv_len)
    _one_device(k, v, q, given, k_pages, v_pages, table, kv_len, freq, q_start, positions)
    rc = lib().apex4_kv_append_rope(qp, qs, heads, op, kp, ks, vp, vs, _starts(q_start, B), T,
                                    None if positions is None else _index(positions, "positions"), fp, rot, _layout(layout),
                                    scale, kpp, vpp, n, tp, width, lp, B, H, D, page, _kind(cache), _stream(k, stream))
    _check("apex4_kv_append_rope", rc)
    return out


def apex4_kv_gather(k_pages, v_pages, table, kv_len, T: int, kv_heads: int, head_dim: int, page: int, q_start=None,
                    cache: str = "fp16", k=None, v=None, stream=None):
    """The last q_start[b + 1] - q_start[b] tokens (None: one) of every sequence
    as float16: (k, v) [T, kv_heads, head_dim]."""
    torch = _torch()
    k = _output(k, (T, kv_heads, head_dim), k_pages, stream)
    v = _output(v, (T, kv_heads, head_dim), k_pages, stream)
    kpp, vpp, n = _planes(k_pages, v_pages, kv_heads, head_dim, page, cache)
    tp, width, lp, B = _tables(table, kv_len)
    rc = lib().apex4_kv_gather(kpp, vpp, n, tp, width, lp, B, kv_heads, head_dim, page, _kind(cache), _starts(q_start, B), T,
                               _ptr(k, torch.float16, "k"), _ptr(v, torch.float16, "v"), _stream(k_pages, stream))
    _check("apex4_kv_gather", rc)
    return k, v


# sizes depend on shapes and the device's compute units alone
@functools.lru_cache(maxsize=1024)
def _decode_need(device, *shape):
    b = ctypes.c_int64(0)
    _check("apex4_attn_decode_workspace_size", lib().apex4_attn_decode_workspace_size(*shape, ctypes.byref(b)))
    return int(b.value)


@functools.lru_cache(maxsize=1024)
def _prefill_need(device, *shape):
    b = ctypes.c_int64(0)
    _check("apex4_attn_prefill_workspace_size", lib().apex4_attn_prefill_workspace_size(*shape, ctypes.byref(b)))
    return int(b.value)


def apex4_attn_decode_workspace_size(B: int, width: int, max_len: int, heads: int, kv_heads: int, head_dim: int, page: int,
                                     window: int = 0, sinks: int = 0) -> int:
    """Bytes of workspace apex4_attn_decode needs on the current device (0: none)."""
    return _decode_need(_torch().cuda.current_device(), B, width, max_len, heads, kv_heads, head_dim, page, window, sinks)


def apex4_attn_prefill_workspace_size(T: int, B: int, max_q: int, width: int, max_len: int, heads: int, kv_heads: int,
                                      head_dim: int, page: int, window: int = 0, sinks: int = 0) -> int:
    """Bytes of workspace apex4_attn_prefill needs on the current device (0: none)."""
    return _prefill_need(_torch().cuda.current_device(), T, B, max_q, width, max_len, heads, kv_heads, head_dim, page,
                         window, sinks)


def apex4_attn_decode(q, k_pages, v_pages, table, kv_len, kv_heads: int, page: int, max_len: int | None = None,
                      cache: str = "fp16", window: int = 0, sinks: int = 0, scale: float | None = None, out=None,
                      workspace=None, stream=None):
    """Attention of one new token a sequence, q [B, heads, head_dim] float16 (rows
    any multiple of 8 apart), over the cache: out [B, heads, head_dim].  max_len:
    a bound of kv_len (None: what the table holds); scale None: head_dim^-1/2."""
    torch = _torch()
    qp, qs = _rows(q, "q")
    B, H, D = q.shape
    kpp, vpp, n = _planes(k_pages, v_pages, kv_heads, D, page, cache)
    tp, width, lp, rows = _tables(table, kv_len)
    if rows != B:
        raise ValueError("q must have one row a sequence")
    most = width * page if max_len is None else max_len
    out = _output_like(out, q, stream)
    need = _decode_need(q.get_device(), B, width, most, H, kv_heads, D, page, window, sinks) if workspace is None else 0
    wp, wn, held = _workspace(workspace, need, q, stream)
    rc = lib().apex4_attn_decode(qp, qs, kpp, vpp, n, tp, width, lp, B, most, H, kv_heads, D, page, _kind(cache), window,
                                 sinks, 1.0 / math.sqrt(D) if scale is None else scale, _ptr(out, torch.float16, "out"), wp,
                                 wn, _stream(q, stream))
    _check("apex4_attn_decode", rc)
    return out


def apex4_attn_prefill(q, q_start, k_pages, v_pages, table, kv_len, kv_heads: int, page: int, max_q: int | None = None,
                       max_len: int | None = None, cache: str = "fp16", window: int = 0, sinks: int = 0,
                       scale: float | None = None, out=None, workspace=None, stream=None):
    """Attention of the packed new tokens q [T, heads, head_dim] of q_start [B + 1]
    over the cache that already holds them: out [T, heads, head_dim].  max_q,
    max_len: bounds of the new and the cached tokens of a sequence."""
    torch = _torch()
    qp, qs = _rows(q, "q")
    T, H, D = q.shape
    kpp, vpp, n = _planes(k_pages, v_pages, kv_heads, D, page, cache)
    tp, width, lp, B = _tables(table, kv_len)
    sp = _starts(q_start, B)
    most = width * page if max_len is None else max_len
    most_q = T if max_q is None else max_q
    out = _output_like(out, q, stream)
    need = (_prefill_need(q.get_device(), T, B, most_q, width, most, H, kv_heads, D, page, window, sinks)
            if workspace is None else 0)
    wp, wn, held = _workspace(workspace, need, q, stream)
    rc = lib().apex4_attn_prefill(qp, qs, sp, T, most_q, kpp, vpp, n, tp, width, lp, B, most, H, kv_heads, D, page,
                                  _kind(cache), window, sinks, 1.0 / math.sqrt(D) if scale is None else scale,
                                  _ptr(out, torch.float16, "out"), wp, wn, _stream(q, stream))
    _check("apex4_attn_prefill", rc)
    return out


@functools.lru_cache(maxsize=256)
def apex4_pages_workspace_size(n_pages: int, n: int) -> int:
    """Bytes of workspace the page calls need for n slots."""
    b = ctypes.c_int64(0)
    _check("apex4_pages_workspace_size", lib().apex4_pages_workspace_size(n_pages, n, ctypes.byref(b)))
    return int(b.value)


def _state(table, kv_len, refs):
    tp, width, lp, slots = _tables(table, kv_len)
    if refs.dim() != 1:
        raise ValueError("refs must be [pages]")
    return tp, slots, width, lp, _index(refs, "refs"), refs.shape[0]


def _pool(pool, refs):
    torch = _torch()
    if pool.dim() != 3 or pool.shape[1] != refs.shape[0]:
        raise ValueError("pool must be [planes, pages, page bytes]")
    return _ptr(pool, torch.uint8, "pool"), pool.shape[0], pool.shape[2]


def _status(status, like, stream):
    if status is None:
        return _empty(like, (1,), _torch().int32, stream)
    if status.numel() < 1:
        raise ValueError("status must be [1]")
    return status


def _pages_work(workspace, n_pages, n, like, stream):
    return _workspace(workspace, 0 if workspace is not None else apex4_pages_workspace_size(n_pages, n), like, stream)


def _same_length(a, b, names):
    if a.dim() != 1 or a.shape != b.shape:
        raise ValueError(f"{names} must be [n] each")
    return a.shape[0]


def apex4_pages_reserve(table, kv_len, refs, seqs, new_len, page: int, status=None, workspace=None, stream=None):
    """Pages for new_len tokens of each of the slots seqs (all or nothing), and
    their kv_len, which counts them whether they are written or not.  Returns status, int32 [1] on the device: 0, > 0 where free
    pages are too few, -1 where a length does not fit the table."""
    args = _state(table, kv_len, refs)
    n = _same_length(seqs, new_len, "seqs and new_len")
    status = _status(status, table, stream)
    wp, wn, held = _pages_work(workspace, args[-1], n, table, stream)
    rc = lib().apex4_pages_reserve(*args, _index(seqs, "seqs"), _index(new_len, "new_len"), n, page,
                                   _index(status, "status"), wp, wn, _stream(table, stream))
    _check("apex4_pages_reserve", rc)
    return status


def apex4_pages_fork(pool, table, kv_len, refs, parents, children, page: int, status=None, workspace=None, stream=None):
    """The (empty) slots children continue parents: full pages shared, a partly
    filled last one copied.  All of a parent's kv_len is taken as written: tokens that
    it only reserved would be written to shared pages by both.  Returns status, int32 [1]: 0, or the pages missing
    (then nothing has changed)."""
    args = _state(table, kv_len, refs)
    pp, planes, size = _pool(pool, refs)
    n = _same_length(parents, children, "parents and children")
    status = _status(status, table, stream)
    wp, wn, held = _pages_work(workspace, args[-1], n, table, stream)
    rc = lib().apex4_pages_fork(pp, planes, size, *args, _index(parents, "parents"), _index(children, "children"), n, page,
                                _index(status, "status"), wp, wn, _stream(table, stream))
    _check("apex4_pages_fork", rc)
    return status


def apex4_pages_free(table, kv_len, refs, seqs, stream=None):
    """Gives back the pages of the slots seqs and empties them."""
    args = _state(table, kv_len, refs)
    if seqs.dim() != 1:
        raise ValueError("seqs must be [n]")
    rc = lib().apex4_pages_free(*args, _index(seqs, "seqs"), seqs.shape[0], _stream(table, stream))
    _check("apex4_pages_free", rc)


def apex4_pages_compact(pool, table, refs, status=None, workspace=None, stream=None):
    """Moves the live pages to the pool's beginning.  Returns status, int32 [1]:
    how many are live."""
    if table.dim() != 2 or refs.dim() != 1:
        raise ValueError("table must be [slots, width] and refs [pages]")
    pp, planes, size = _pool(pool, refs)
    status = _status(status, table, stream)
    wp, wn, held = _pages_work(workspace, refs.shape[0], 0, table, stream)
    rc = lib().apex4_pages_compact(pp, planes, size, _index(table, "table"), table.shape[0], table.shape[1],
                                   _index(refs, "refs"), refs.shape[0], _index(status, "status"), wp, wn,
                                   _stream(table, stream))
    _check("apex4_pages_compact", rc)
    return status


def apex4_pages_copy(pool, src, dst, stream=None):
    """Page src[i] to dst[i] in every plane of pool [planes, pages, page bytes]."""
    torch = _torch()
    n = _same_length(src, dst, "src and dst")
    if pool.dim() != 3:
        raise ValueError("pool must be [planes, pages, page bytes]")
    rc = lib().apex4_pages_copy(_dev(pool, torch.uint8, "pool"), pool.shape[0], pool.shape[2], pool.shape[1],
                                _index(src, "src"), _index(dst, "dst"), n, _stream(pool, stream))
    _check("apex4_pages_copy", rc)


class PagedKVCache:
    """The planes of all layers, the page tables of ``slots`` sequences and the
    pages' reference counts.  Everything stays on the device: with slots and lengths
    given as device tensors no call waits for it, so a step can be captured into a
    HIP graph; a list is copied there first, which waits for the stream's work and
    cannot be captured.  reserve and fork return their outcome as a device tensor
    (``reserved(status)`` reads it).

    pages: of each plane; page: tokens a page; max_len: tokens a sequence may
    reach, to the end of the page that holds the last (kept so as ``max_len``)."""

    def __init__(self, layers: int, pages: int, slots: int, kv_heads: int, head_dim: int = 128, page: int = 16,
                 max_len: int = 4096, cache: str = "fp16", device="cuda"):
        torch = _torch()
        size = apex4_kv_page_bytes(cache, kv_heads, head_dim, page)
        self.layers, self.kv_heads, self.head_dim, self.page, self.cache = layers, kv_heads, head_dim, page, cache
        width = -(-max_len // page)
        self.max_len = width * page  # what reserve gives, and so what attention has to see
        self.pool = torch.zeros((2 * layers, pages, size), dtype=torch.uint8, device=device)
        self.table = torch.full((slots, width), -1, dtype=torch.int32, device=device)
        self.kv_len = torch.zeros((slots,), dtype=torch.int32, device=device)
        self.refs = torch.zeros((pages,), dtype=torch.int32, device=device)
        self.planes = [(self.pool[2 * i], self.pool[2 * i + 1]) for i in range(layers)]

    def _seqs(self, seqs, stream=None):
        """A list as a tensor of the stream that the call runs on: its memory goes
        to no other call before that stream has read it."""
        torch = _torch()
        if isinstance(seqs, torch.Tensor):
            return seqs
        with torch.cuda.stream(stream):  # None: the current one
            return torch.tensor(seqs, dtype=torch.int32, device=self.table.device)

    @staticmethod
    def reserved(status) -> bool:
        """Whether a reserve or fork had its pages (waits for the device)."""
        return int(status.item()) == 0

    def reserve(self, seqs, new_len, **kw):
        return apex4_pages_reserve(self.table, self.kv_len, self.refs, self._seqs(seqs, kw.get("stream")),
                                   self._seqs(new_len, kw.get("stream")), self.page, **kw)

    def fork(self, parents, children, **kw):
        return apex4_pages_fork(self.pool, self.table, self.kv_len, self.refs, self._seqs(parents, kw.get("stream")),
                                self._seqs(children, kw.get("stream")), self.page, **kw)

    def free(self, seqs, **kw):
        apex4_pages_free(self.table, self.kv_len, self.refs, self._seqs(seqs, kw.get("stream")), **kw)

    def compact(self, **kw):
        return apex4_pages_compact(self.pool, self.table, self.refs, **kw)

    def batch(self, seqs):
        """(table rows, lengths) of the sequences of one step."""
        i = self._seqs(seqs).long()
        return self.table[i], self.kv_len[i]

    def append(self, layer, k, v, batch, q_start=None, **kw):
        apex4_kv_append(k, v, *self.planes[layer], *batch, self.page, q_start=q_start, cache=self.cache, **kw)

    def append_rope(self, layer, q, k, v, batch, freq, q_start=None, **kw):
        return apex4_kv_append_rope(q, k, v, *self.planes[layer], *batch, self.page, freq, q_start=q_start, cache=self.cache, **kw)

    def gather(self, layer, T, batch, q_start=None, **kw):
        return apex4_kv_gather(*self.planes[layer], *batch, T, self.kv_heads, self.head_dim, self.page, q_start=q_start,
                               cache=self.cache, **kw)

    def decode(self, layer, q, batch, **kw):
        return apex4_attn_decode(q, *self.planes[layer], *batch, self.kv_heads, self.page,
                                 **{"max_len": self.max_len, "cache": self.cache, **kw})

    def prefill(self, layer, q, batch, q_start, max_q, **kw):
        return apex4_attn_prefill(q, q_start, *self.planes[layer], *batch, self.kv_heads, self.page, max_q=max_q,
                                  **{"max_len": self.max_len, "cache": self.cache, **kw})
