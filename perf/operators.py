"""The operators of a paged key-value cache, measured through the framework's
public entry points: attention over the cache for single new tokens and for
chunks of prompts, with or without a sliding window and a few first tokens that
stay visible, writing and reading tokens, and the cache's pages.

A plane of a cache (the keys, or the values, of one layer) is uint8
[pages, page bytes].  A page of a "fp16" cache holds [kv heads][page][D]
binary16; one of an "int4" cache holds codes [kv heads][page][D/2] (two signed
codes a byte, low nibble first) and then binary16 scales [kv heads][page], one
for a token's D values (SymQuant with G = D).  Token t of sequence b lies in
page table[b][t / page].

Kinds of case
  append   the keys and values of new tokens written into a cache, read back
           as the values that it now holds
  decode   one new token a sequence attends to the cache
  prefill  several new tokens a sequence, already in the cache, attend to it:
           a token at position p sees the positions up to p
  fork     a beam step: every beam continues one of the beams before it (full
           pages shared, the last one copied), then the beams before are freed
  churn    a batch ends: its pages are freed, the cache is compacted, and the
           next batch's pages are reserved

With a window w > 0, position p sees only p - w + 1 .. p and the first `sinks`
positions.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def listed():
    return [
        # one decode step's tokens into the cache of a Llama-2-70B layer: the smallest call, launches and host time
        {"name": "append_step", "kind": "append", "B": 16, "new": 1, "len": 2000, "Hkv": 8, "D": 128, "page": 16, "cache": "fp16", "ragged": True},
        # prompts of several lengths quantized into a 4-bit cache
        {"name": "append_prompts_int4", "kind": "append", "B": 5, "new": 4001, "len": 4001, "Hkv": 8, "D": 128, "page": 64, "cache": "int4", "ragged": True},
        # single-stream decode early in a conversation, Llama-2-70B heads
        {"name": "decode_1", "kind": "decode", "B": 1, "len": 517, "Hq": 64, "Hkv": 8, "D": 128, "page": 16, "cache": "fp16", "window": 0, "sinks": 0, "ragged": False},
        # a server's decode batch, sequences of all lengths
        {"name": "decode_batch", "kind": "decode", "B": 27, "len": 8192, "Hq": 64, "Hkv": 8, "D": 128, "page": 16, "cache": "fp16", "window": 0, "sinks": 0, "ragged": True},
        # one very long document
        {"name": "decode_long", "kind": "decode", "B": 1, "len": 131071, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "cache": "fp16", "window": 0, "sinks": 0, "ragged": False},
        # the same server with the cache in 4 bits
        {"name": "decode_batch_int4", "kind": "decode", "B": 32, "len": 16384, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "cache": "int4", "window": 0, "sinks": 0, "ragged": True},
        # endless streams: a window and four first tokens, one head each
        {"name": "decode_window", "kind": "decode", "B": 16, "len": 16384, "Hq": 40, "Hkv": 40, "D": 128, "page": 32, "cache": "fp16", "window": 2048, "sinks": 4, "ragged": True},
        # a whole prompt: the largest call
        {"name": "prefill_prompt", "kind": "prefill", "B": 1, "new": 8192, "len": 8192, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "cache": "fp16", "window": 0, "sinks": 0, "ragged": False},
        # chunks of several prompts behind what the cache holds of them, small heads
        {"name": "prefill_chunks", "kind": "prefill", "B": 6, "new": 700, "len": 4096, "Hq": 40, "Hkv": 8, "D": 64, "page": 16, "cache": "fp16", "window": 0, "sinks": 0, "ragged": True},
        # a chunk of a long stream under a window, 4-bit cache
        {"name": "prefill_window_int4", "kind": "prefill", "B": 2, "new": 2048, "len": 8192, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "cache": "int4", "window": 1024, "sinks": 4, "ragged": False},
        # beam search, 8 requests of 4 beams
        {"name": "fork_beams", "kind": "fork", "B": 8, "beams": 4, "len": 1000, "layers": 6, "Hkv": 8, "D": 128, "page": 16, "cache": "fp16"},
        # a server's batch turns over
        {"name": "churn_batch", "kind": "churn", "B": 24, "len": 2048, "layers": 4, "Hkv": 8, "D": 128, "page": 16, "cache": "fp16"},
    ]


MOST_SCORES = 8192 * 8192 * 64  # score matrix of the largest listed case
MOST_BYTES = 1 << 29


def _log(rng, lo, hi):
    return round(lo * (hi / lo) ** rng.random())


def draw(rng):
    kind = rng.choices(["append", "decode", "prefill", "fork", "churn"], [2, 5, 4, 1, 1])[0]
    while True:
        Hkv = rng.choice([1, 2, 4, 5, 8, 8, 8, 40])
        c = {"kind": kind, "B": _log(rng, 1, 48), "Hkv": Hkv, "D": rng.choice([64, 128, 128, 128]),
             "page": rng.choice([16, 16, 32, 64, 128]), "cache": rng.choice(["fp16", "fp16", "int4"])}
        token = Hkv * c["D"] * 4  # bytes a token of a binary16 cache takes
        if kind in ("fork", "churn"):
            c |= {"len": _log(rng, 40, 4000), "layers": _log(rng, 1, 32)}
            if kind == "fork":
                c |= {"B": _log(rng, 1, 12), "beams": rng.randint(2, 8)}
            if 2 * c["B"] * c.get("beams", 1) * (c["len"] + c["page"]) * token * c["layers"] <= 4 * MOST_BYTES:
                return c
            continue
        c |= {"ragged": rng.random() < 0.6}
        if kind == "append":
            c |= {"new": 1 if rng.random() < 0.4 else _log(rng, 2, 4096)}
            c |= {"len": c["new"] + _log(rng, 1, 2000)}
            if c["B"] * c["len"] * token <= MOST_BYTES:
                return c
            continue
        c |= {"Hq": Hkv * (1 if Hkv == 40 else rng.choice([1, 2, 4, 5, 7, 8, 16])), "window": 0, "sinks": 0}
        if rng.random() < 0.4:
            c |= {"window": _log(rng, 16, 8192), "sinks": rng.choice([0, 1, 4, 4, 64])}
        c |= {"len": _log(rng, 16, 131072 if kind == "decode" else 8192)}
        if kind == "decode":
            if c["B"] * c["len"] * token <= MOST_BYTES and c["Hq"] <= 128:
                return c
            continue
        c |= {"new": _log(rng, 1, c["len"]) if rng.random() < 0.7 else c["len"]}
        if c["B"] * c["Hq"] * c["new"] * c["len"] <= MOST_SCORES // 2 and c["B"] * c["len"] * token <= MOST_BYTES and c["Hq"] <= 128:
            return c


# ---------------------------------------------------------------- lengths


def _lengths(case):
    """(cached tokens with the new ones, new tokens) of every sequence: what a
    scheduler knows on the host."""
    B, most, new = case["B"], case["len"], case.get("new", 1)
    if not case.get("ragged"):
        return [most] * B, [new] * B
    rng = random.Random("%d %d %d" % (B, most, new))
    news = [new if new == 1 else rng.randint(1, new) for _ in range(B)]
    lens = [max(n, rng.randint(max(1, most // 16), most)) for n in news]
    lens[0], news[0] = most, new
    if B > 4 and case["kind"] == "decode":
        lens[B // 2] = 0  # a slot of the batch that is idle
    return lens, news


def _batch_lengths(case, n):
    rng = random.Random("%d %d" % (n, case["len"]))
    return [rng.randint(max(1, case["len"] // 2), case["len"]) for _ in range(n)]


def _pages(tokens, page):
    return -(-tokens // page)


def _page_bytes(case):
    n = case["Hkv"] * case["page"]
    return n * case["D"] * 2 if case["cache"] == "fp16" else n * (case["D"] // 2 + 2)


# ---------------------------------------------------------------- inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _plane(case, pages, g):
    """One plane with every page filled: values of about unit size."""
    n, D = case["Hkv"] * case["page"], case["D"]
    if case["cache"] == "fp16":
        x = torch.empty((pages, n * D), dtype=torch.float16, device="cuda").normal_(0.0, 1.0, generator=g)
        return x.view(torch.uint8)
    codes = torch.randint(0, 256, (pages, n * D // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = (torch.rand((pages, n), device="cuda", generator=g) * 0.2 + 0.1).to(torch.float16)
    return torch.cat((codes, scales.view(torch.uint8)), dim=1)


def _table(rows, pages, width, g):
    """Page tables of sequences of rows[i] pages over randomly ordered pages; -1 where there is none."""
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(rows), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(rows):
        table[i, :n] = order[at:at + n]
        at += n
    return table


def _tokens(T, heads, D, g, std):
    """[T, heads, D] out of the wider rows of a fused projection."""
    wide = torch.empty((T, heads * D + 256), dtype=torch.float16, device="cuda").normal_(0.0, std, generator=g)
    return wide[:, 128:128 + heads * D].view(T, heads, D)


def prepare(case, seed):
    g = _gen(seed)
    kind, page = case["kind"], case["page"]
    if kind in ("fork", "churn"):
        return _prepare_pages(case, g)
    lens, news = _lengths(case)
    rows = [_pages(n, page) for n in lens]
    pages = sum(rows) + 3
    start = [0]
    for n in news:
        start.append(start[-1] + n)
    s = {"case": case, "k_pages": _plane(case, pages, g), "v_pages": _plane(case, pages, g),
         "table": _table(rows, pages, max(rows) + 1, g), "kv_len": _ints(lens), "q_start": _ints(start),
         "max_len": max(lens), "max_q": max(news), "T": start[-1], "one": max(news) == 1}
    if kind == "append":
        s["k"] = _tokens(s["T"], case["Hkv"], case["D"], g, 1.0)
        s["v"] = _tokens(s["T"], case["Hkv"], case["D"], g, 1.0)
        # a binary16 cache is returned whole beside what is read back of it
        s["held"] = tuple(s[x].view(torch.float16) for x in ("k_pages", "v_pages")) if case["cache"] == "fp16" else ()
    else:
        s["q"] = _tokens(s["T"], case["Hq"], case["D"], g, 1.5)
    return s


def _prepare_pages(case, g):
    page, n = case["page"], case["B"] * case.get("beams", 1)
    lens = _batch_lengths(case, n)
    rows = [_pages(x, page) for x in lens]
    if case["kind"] == "fork":
        pages, slots = sum(rows) + 2 * n, 2 * n
        parents = torch.arange(n, device="cuda") // case["beams"] * case["beams"]
        parents = parents + torch.randint(0, case["beams"], (n,), device="cuda", generator=g)
        here, there = torch.arange(n, device="cuda"), torch.arange(n, 2 * n, device="cuda")
        s = {"parents": parents.to(torch.int32), "halves": [here.to(torch.int32), there.to(torch.int32)],
             "from": [parents.to(torch.int32), (parents + n).to(torch.int32)]}
        table = _table(rows + [0] * n, pages, max(rows) + 1, g)
        kv_len = _ints(lens + [0] * n)
    else:  # two batches, in turn
        other = _batch_lengths({"len": case["len"] - 7}, n)
        rows2 = [_pages(x, page) for x in other]
        pages, slots = sum(rows) + sum(rows2) + 5, 2 * n
        s = {"halves": [_ints(list(range(n))), _ints(list(range(n, 2 * n)))], "lens": [_ints(lens), _ints(other)]}
        table = _table(rows + rows2, pages, max(rows + rows2) + 1, g)
        kv_len = _ints(lens + other)
    used = table[table >= 0].long()
    refs = torch.zeros((pages,), dtype=torch.int32, device="cuda")
    refs[used] = 1
    pool = torch.stack([_plane(case, pages, g) for _ in range(2 * case["layers"])])
    return s | {"case": case, "pool": pool, "table": table, "kv_len": kv_len, "refs": refs, "turn": 0}


# ---------------------------------------------------------------- one pass


def run(state):
    return (_framework if own else _plain)(state)


def _framework(s):
    import paper_2606_08761_amd as apex4
    c = s["case"]
    kind = c["kind"]
    if kind in ("fork", "churn"):
        now = s["turn"]
        s["turn"] = 1 - now
        if kind == "fork":
            apex4.apex4_pages_fork(s["pool"], s["table"], s["kv_len"], s["refs"], s["from"][now], s["halves"][1 - now], c["page"])
            apex4.apex4_pages_free(s["table"], s["kv_len"], s["refs"], s["halves"][now])
        else:
            apex4.apex4_pages_free(s["table"], s["kv_len"], s["refs"], s["halves"][now])
            apex4.apex4_pages_compact(s["pool"], s["table"], s["refs"])
            apex4.apex4_pages_reserve(s["table"], s["kv_len"], s["refs"], s["halves"][now], s["lens"][now], c["page"])
        return s["pool"], s["table"], s["kv_len"], s["refs"]
    start = None if s["one"] else s["q_start"]
    if kind == "append":
        apex4.apex4_kv_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], c["page"],
                              q_start=start, cache=c["cache"])
        return apex4.apex4_kv_gather(s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["T"], c["Hkv"], c["D"], c["page"],
                                     q_start=start, cache=c["cache"]) + s["held"]
    if kind == "decode":
        return apex4.apex4_attn_decode(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], c["Hkv"], c["page"],
                                       max_len=s["max_len"], cache=c["cache"], window=c["window"], sinks=c["sinks"])
    return apex4.apex4_attn_prefill(s["q"], s["q_start"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], c["Hkv"], c["page"],
                                    max_q=s["max_q"], max_len=s["max_len"], cache=c["cache"], window=c["window"], sinks=c["sinks"])


# ---------------------------------------------------------------- the plain forms


def _split(pages, case):
    """Views of a plane: binary16 values [P, Hkv, page, D], or codes [P, Hkv, page, D/2] and scales [P, Hkv, page]."""
    P, H, page, D = pages.shape[0], case["Hkv"], case["page"], case["D"]
    if case["cache"] == "fp16":
        return pages.view(torch.float16).view(P, H, page, D), None
    n = H * page * D // 2
    return pages[:, :n].unflatten(1, (H, page, D // 2)), pages[:, n:].view(torch.float16).unflatten(1, (H, page))


def _values(x, scales):
    """float32 values of what _split gave, indexed alike."""
    if scales is None:
        return x.float()
    low = (x & 15).to(torch.int8)
    high = (x >> 4).to(torch.int8)
    n = torch.stack((low, high), dim=-1).flatten(-2)
    return torch.where(n > 7, n - 16, n).float() * scales.float()[..., None]


def _dense(pages, table, case):
    """[B, Hkv, positions, D] float32."""
    x, scales = _split(pages, case)
    at = table.clamp(min=0).long()
    v = _values(x[at], None if scales is None else scales[at])
    return v.transpose(1, 2).flatten(2, 3)


def _where(s):
    """The sequence of every new token, and its position."""
    T = s["T"]
    start, tok = s["q_start"].long(), torch.arange(T, device="cuda")
    seq = torch.searchsorted(start, tok, right=True) - 1
    pos = s["kv_len"].long()[seq] - start[seq + 1] + tok
    return seq, pos


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "fork":
        return _plain_fork(s)
    if kind == "churn":
        return _plain_churn(s)
    return _plain_append(s) if kind == "append" else _plain_attention(s)


def _plain_append(s):
    c = s["case"]
    seq, pos = _where(s)
    page = s["table"][seq, pos // c["page"]].long()
    return tuple(_plain_write(s[x], s[x + "_pages"], page, pos % c["page"], c) for x in ("k", "v")) + s["held"]


def _plain_write(x, pages, page, off, c):
    into, scales = _split(pages, c)
    if scales is None:
        into[page, :, off] = x
    else:
        v = x.float()
        sc = (v.abs().amax(dim=2) / 7.0).to(torch.float16)
        q = torch.where(sc[..., None] > 0, v / sc.float()[..., None], torch.zeros_like(v)).round().clamp(-8, 7)
        n = q.to(torch.int8).view(torch.uint8) & 15
        into[page, :, off] = n[..., 0::2] | (n[..., 1::2] << 4)
        scales[page, :, off] = sc
        scales = scales[page, :, off]
    return _values(into[page, :, off], scales).to(torch.float16)


def _plain_attention(s):
    """Every sequence's new tokens padded to the most, scores over all positions of the table."""
    c = s["case"]
    B, Hq, H, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    q, n = s["q"].float() / math.sqrt(D), s["max_q"]
    seq, pos = _where(s)
    start, lens = s["q_start"].long(), s["kv_len"].long()
    row = torch.arange(s["T"], device="cuda") - start[seq]
    padded = torch.zeros((B, n, Hq, D), device="cuda")
    padded[seq, row] = q
    k, v = _dense(s["k_pages"], s["table"], c), _dense(s["v_pages"], s["table"], c)
    x = padded.view(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D) @ k.transpose(2, 3)
    x = x.view(B, H, Hq // H, n, -1)
    at = torch.arange(x.shape[-1], device="cuda")
    p = (lens - (start[1:] - start[:-1]))[:, None] + torch.arange(n, device="cuda")  # position of every row
    seen = (at <= p[..., None]) & (at < lens[:, None, None])
    if c["window"]:
        seen &= (at > p[..., None] - c["window"]) | (at < c["sinks"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x -= x.amax(dim=-1, keepdim=True).clamp(min=-1e38)
    x.exp_()
    total = x.sum(dim=-1, keepdim=True)
    y = (x.view(B, H, -1, x.shape[-1]) @ v).view(B, H, Hq // H, n, D)
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    return y.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[seq, row].to(torch.float16)


def _plain_free(s, seqs):
    rows = s["table"][seqs.long()]
    held = rows >= 0
    s["refs"].index_add_(0, rows.clamp(min=0).flatten().long(), -held.flatten().to(torch.int32))
    s["table"][seqs.long()] = -1
    s["kv_len"][seqs.long()] = 0


def _lowest_free(refs):
    """All pages, the free ones first, each group in ascending order."""
    return torch.argsort((refs > 0).to(torch.int8), stable=True).to(torch.int32)


def _plain_fork(s):
    c, now = s["case"], s["turn"]
    s["turn"] = 1 - now
    old, new, parents = s["halves"][now], s["halves"][1 - now].long(), s["from"][now].long()
    table, refs, page = s["table"], s["refs"], c["page"]
    lens = s["kv_len"][parents]
    rows = table[parents]
    last, part = (lens // page).long(), lens % page != 0
    rank = torch.cumsum(part.to(torch.int64), 0) - 1
    fresh = _lowest_free(refs)[rank.clamp(min=0)]
    which = torch.arange(len(new), device="cuda")
    src = rows[which, last.clamp(max=rows.shape[1] - 1)]
    child = rows.clone()
    child[which, last.clamp(max=rows.shape[1] - 1)] = torch.where(part, fresh, src)
    refs.index_add_(0, child.clamp(min=0).flatten().long(), (child >= 0).flatten().to(torch.int32))
    table[new] = child
    s["kv_len"][new] = lens
    pairs = part.nonzero().flatten()
    s["pool"][:, fresh[pairs].long()] = s["pool"][:, src[pairs].long()]
    _plain_free(s, old)
    return s["pool"], table, s["kv_len"], refs


def _plain_churn(s):
    c, now = s["case"], s["turn"]
    s["turn"] = 1 - now
    table, refs, page = s["table"], s["refs"], c["page"]
    seqs, lens = s["halves"][now], s["lens"][now]
    _plain_free(s, seqs)
    # compact: the live pages past the number of live ones go to the free ones before it
    live = refs > 0
    number = torch.arange(len(refs), device="cuda")
    low = number < live.sum()
    src, dst = (live & ~low).nonzero().flatten(), (~live & low).nonzero().flatten()
    to = number.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s["pool"][:, dst] = s["pool"][:, src]
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    # reserve: the lowest free pages, in the order of the sequences
    need = (lens + page - 1) // page
    first = torch.cumsum(need, 0) - need
    column = torch.arange(table.shape[1], device="cuda")
    mine = column < need[:, None]
    order = _lowest_free(refs)
    got = order[torch.where(mine, first[:, None] + column, torch.zeros_like(column)).long()]
    table[seqs.long()] = torch.where(mine, got, torch.full_like(got, -1))
    refs.index_add_(0, got.flatten().long(), mine.flatten().to(torch.int32))
    s["kv_len"][seqs.long()] = lens
    return s["pool"], table, s["kv_len"], refs


# ---------------------------------------------------------------- what a pass cannot do without


def _seen(case, length, new):
    """Pairs (new token, position it sees), and the positions that any of them sees."""
    w, sinks = case["window"], case["sinks"]
    if not w:
        return sum(range(length - new + 1, length + 1)), length
    pairs = 0
    for p in range(length - new, length):
        lo = max(0, p - w + 1)
        pairs += p + 1 - lo + min(sinks, lo)
    lo = max(0, length - new - w + 1)
    return pairs, length - lo + min(sinks, lo)


def work(case):
    kind = case["kind"]
    token = 2 * case["Hkv"] * (case["D"] * 2 if case["cache"] == "fp16" else case["D"] // 2 + 2)  # keys and values
    if kind == "fork":
        n = case["B"] * case["beams"]
        lens = _batch_lengths(case, n)
        part = sum(x % case["page"] != 0 for x in lens)
        held = sum(_pages(x, case["page"]) for x in lens)
        return {"bytes": 2 * part * 2 * case["layers"] * _page_bytes(case) + 24 * held, "flops": 0}
    if kind == "churn":
        a, b = _batch_lengths(case, case["B"]), _batch_lengths({"len": case["len"] - 7}, case["B"])
        pages = min(sum(_pages(x, case["page"]) for x in y) for y in (a, b))
        return {"bytes": 2 * pages * 2 * case["layers"] * _page_bytes(case) + 24 * pages, "flops": 0}
    lens, news = _lengths(case)
    if kind == "append":  # the tokens read, the cache written and read, the values written
        return {"bytes": sum(news) * (2 * token + 8 * case["Hkv"] * case["D"]), "flops": 0}
    pairs, seen = 0, 0
    for a, b in zip(lens, news):
        x = _seen(case, a, min(a, b))
        pairs, seen = pairs + x[0], seen + x[1]
    return {"bytes": seen * token + 4 * sum(news) * case["Hq"] * case["D"], "flops": 4.0 * pairs * case["Hq"] * case["D"]}


# ---------------------------------------------------------------- 64 bits


def exact(case, seed):
    if case["kind"] in ("fork", "churn"):
        return None  # moves and whole numbers
    s = prepare(case, seed)
    if case["kind"] == "append":
        return tuple(_exact_stored(s[x], case) for x in ("k", "v")) + (None,) * len(s["held"])
    lens, news = _lengths(case)
    out = torch.zeros((s["T"], case["Hq"], case["D"]), dtype=torch.float64, device="cuda")
    at = 0
    for b, (length, new) in enumerate(zip(lens, news)):
        if length:
            ids = s["table"][b, :_pages(length, case["page"])].long()
            for h in range(case["Hkv"]):
                k, v = (_exact_rows(s[x], ids, h, case)[:length] for x in ("k_pages", "v_pages"))
                _exact_rows_of_head(s["q"], k, v, out, at, new, h, case)
        at += new
    return out


def _exact_stored(x, case):
    v = x.double()
    if case["cache"] == "fp16":
        return v
    sc = (v.abs().amax(dim=-1, keepdim=True) / 7.0).to(torch.float16).double()
    return torch.where(sc > 0, (v / sc).round().clamp(-8, 7) * sc, torch.zeros_like(v))


def _exact_rows(pages, ids, h, case):
    page, D = case["page"], case["D"]
    x = pages[ids]
    if case["cache"] == "fp16":
        return x.view(torch.float16)[:, h * page * D:(h + 1) * page * D].reshape(-1, D).double()
    codes = x[:, h * page * D // 2:(h + 1) * page * D // 2].reshape(-1, D // 2).to(torch.int32)
    at = case["Hkv"] * page * D // 2 + 2 * h * page
    scales = x[:, at:at + 2 * page].contiguous().view(torch.float16).reshape(-1, 1).double()
    v = torch.empty((codes.shape[0], D), dtype=torch.float64, device="cuda")
    v[:, 0::2] = ((codes & 15) ^ 8) - 8.0
    v[:, 1::2] = ((codes >> 4) ^ 8) - 8.0
    return v * scales


def _exact_rows_of_head(q, k, v, out, at, new, h, case):
    """The rows of one sequence and key head, 1024 new tokens at a time."""
    group, length = case["Hq"] // case["Hkv"], k.shape[0]
    heads = slice(h * group, (h + 1) * group)
    t = torch.arange(length, device="cuda")
    for i in range(0, new, 1024):
        n = min(1024, new - i)
        p = length - new + i + torch.arange(n, device="cuda")[:, None]
        seen = t <= p
        if case["window"]:
            seen = seen & ((p - t < case["window"]) | (t < case["sinks"]))
        x = q[at + i:at + i + n, heads].double().reshape(n * group, -1) @ k.t().contiguous()
        x = x.view(n, group, length) / math.sqrt(case["D"])
        x = torch.where(seen[:, None], x, torch.full_like(x, -math.inf))
        y = torch.softmax(x, dim=-1).view(n * group, length) @ v
        out[at + i:at + i + n, heads] = y.view(n, group, -1)
