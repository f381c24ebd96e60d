"""The operators that take a decoder from its projections to its next tokens,
measured through the framework's public entry points: rotary positions, the same on
the way into a paged key-value cache, linears in 8 bits, and the choice of a token.

Kinds of case
  rope    the first `rot` values of every head of a token turned by its position
  append  new tokens' queries and keys turned, keys and values written into a paged
          cache (layout as in perf/operators.py); from a 4-bit cache read back as the
          values that it now holds
  linear  x quantized to 8 bits a token, times weights in 8 bits with a scale a channel
  sample  a token for every row of logits: temperature, top-k, top-p, min-p, and one
          given random number

Rotary positions.  Pair j < rot/2 of a token at position p turns by p freq[j] whole
turns (freq is binary64, so far positions keep their angle), times `mag`:
  (a, b) -> mag (a cos - b sin, b cos + a sin),
the pair being (j, j + rot/2) in the "half" layout and (2j, 2j + 1) in the
"interleaved" one.

8 bits.  Codes clamp(round(x / s), -127, 127), s = binary32(max|x| / 127) of a token;
y = s_token s_channel sum(codes codes).

Sampling.  w = exp((x - max) / temperature), in the order of falling logits, equal ones
by index.  top-k keeps the first k; top-p of these the shortest beginning that holds p
of their sum; min-p those with w >= min_p.  The token is the first, by index, whose
running sum of kept weights passes u times their sum; its share of that sum is returned
too.  A temperature of zero takes the largest logit.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def listed():
    return [
        # one decode step's queries and keys of a Llama-2-70B layer: the smallest call, launch and host time
        {"name": "rope_step", "kind": "rope", "T": 16, "heads": 72, "D": 128, "rot": 128, "layout": "half", "scaling": "none", "first": 2000},
        # a long prompt's, far into a context that was stretched band by band
        {"name": "rope_prompt", "kind": "rope", "T": 8192, "heads": 72, "D": 128, "rot": 128, "layout": "half", "scaling": "bands", "first": 120000},
        # neighbouring pairs, half of a small head
        {"name": "rope_partial", "kind": "rope", "T": 4001, "heads": 40, "D": 64, "rot": 32, "layout": "interleaved", "scaling": "none", "first": 0},
        # a decode step of a server's batch
        {"name": "append_rope_step", "kind": "append", "B": 16, "new": 1, "len": 2000, "Hq": 64, "Hkv": 8, "D": 128, "rot": 128, "layout": "half", "scaling": "none", "page": 16, "cache": "fp16", "ragged": True},
        # prompts of several lengths into a 4-bit cache, stretched context
        {"name": "append_rope_prompts", "kind": "append", "B": 5, "new": 4001, "len": 4001, "Hq": 64, "Hkv": 8, "D": 128, "rot": 128, "layout": "half", "scaling": "yarn", "page": 64, "cache": "int4", "ragged": True},
        # single-stream decode, an output projection
        {"name": "linear_token", "kind": "linear", "M": 1, "N": 8192, "K": 8192},
        # a server's batch through the widest layer
        {"name": "linear_batch", "kind": "linear", "M": 27, "N": 57344, "K": 8192},
        # a chunk of a prompt beside the batch's tokens
        {"name": "linear_chunk", "kind": "linear", "M": 300, "N": 10240, "K": 8192},
        # a prompt: the largest product
        {"name": "linear_prompt", "kind": "linear", "M": 4096, "N": 10240, "K": 8192},
        # one stream's next token
        {"name": "sample_one", "kind": "sample", "B": 1, "V": 32000, "type": "fp16", "rows": "top-p", "masked": False},
        # a server's batch, every request with its own settings
        {"name": "sample_batch", "kind": "sample", "B": 48, "V": 32000, "type": "fp16", "rows": "mixed", "masked": False},
        # many samples over a large vocabulary, logits that were corrected in 32 bits, tokens masked out
        {"name": "sample_wide", "kind": "sample", "B": 256, "V": 131072, "type": "fp32", "rows": "top-p", "masked": True},
    ]


MOST_VALUES = 8192 * 72 * 128  # of the largest rope case
MOST_BYTES = 1 << 29
MOST_PRODUCTS = 4096 * 10240 * 8192
MOST_LOGITS = 256 * 131072


def _log(rng, lo, hi):
    return round(lo * (hi / lo) ** rng.random())


def _rotary(rng):
    D = rng.choice([64, 128, 128])
    return {"D": D, "rot": rng.choice([D, D, D, D // 2, D // 4]), "layout": rng.choice(["half", "half", "interleaved"]),
            "scaling": rng.choice(["none", "linear", "yarn", "bands"])}


def draw(rng):
    kind = rng.choices(["rope", "append", "linear", "sample"], [2, 2, 4, 3])[0]
    while True:
        if kind == "rope":
            c = {"kind": kind, "T": _log(rng, 1, 16384), "heads": rng.choice([1, 5, 8, 40, 64, 72, 96])} | _rotary(rng)
            c["first"] = rng.choice([0, rng.randint(1, 4096), rng.randint(4097, 1000000)])
            if c["T"] * c["heads"] * c["D"] <= MOST_VALUES:
                return c
        elif kind == "append":
            H = rng.choice([1, 2, 4, 5, 8, 8, 8, 40])
            c = {"kind": kind, "B": _log(rng, 1, 48), "Hkv": H, "Hq": H * (1 if H == 40 else rng.choice([1, 4, 7, 8])), "ragged": rng.random() < 0.6,
                 "page": rng.choice([16, 16, 32, 64, 128]), "cache": rng.choice(["fp16", "fp16", "int4"])} | _rotary(rng)
            c["new"] = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
            c["len"] = c["new"] + _log(rng, 1, 2000)
            if c["B"] * c["len"] * H * c["D"] * 4 <= MOST_BYTES and c["B"] * c["new"] * c["Hq"] * c["D"] <= MOST_VALUES:
                return c
        elif kind == "linear":
            c = {"kind": kind, "M": _log(rng, 1, 8192), "N": rng.choice([8192, 10240, 28672, 32000, 57344, _log(rng, 64, 16384)]),
                 "K": rng.choice([4096, 8192, 8192, 28672, 32 * _log(rng, 8, 512)])}
            if c["N"] * c["K"] <= 57344 * 8192 and c["M"] * c["N"] * c["K"] <= MOST_PRODUCTS:
                return c
        else:
            c = {"kind": kind, "B": _log(rng, 1, 300), "V": rng.choice([32000, 32001, 65536, 131072, _log(rng, 1000, 131072)]),
                 "type": rng.choice(["fp16", "fp16", "fp32"]), "rows": rng.choice(["top-p", "top-k", "plain", "mixed", "mixed"]),
                 "masked": rng.random() < 0.3}
            if c["B"] * c["V"] <= MOST_LOGITS:
                return c


# ---------------------------------------------------------------- inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(shape, g, std=1.0, dtype=torch.float16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _frequencies(case):
    """Whole turns a position, binary64 [rot/2], and the magnitude."""
    n = case["rot"] // 2
    j = torch.arange(n, dtype=torch.float64)
    f = 10000.0 ** (-j / n) / (2 * math.pi)
    kind, factor, trained = case["scaling"], 8.0, 8192.0
    if kind == "linear":
        return (f / factor).cuda(), 1.0
    if kind == "yarn":  # from pairs that turn 32 times in the trained length (kept) to those that turn once (stretched)
        at = [n * math.log(trained / (turns * 2 * math.pi)) / math.log(10000.0) for turns in (32.0, 1.0)]
        keep = 1.0 - ((j - at[0]) / (at[1] - at[0])).clamp(0.0, 1.0)
        return (f * keep + f / factor * (1 - keep)).cuda(), 0.1 * math.log(factor) + 1.0
    if kind == "bands":  # the same by the turns themselves, from 4 (kept) to 1 (stretched)
        keep = ((f * trained - 1.0) / 3.0).clamp(0.0, 1.0)
        return (f * keep + f / factor * (1 - keep)).cuda(), 1.0
    return f.cuda(), 1.0


def _rows(T, heads, D, g):
    """[T, heads, D] out of the wider rows of a fused projection."""
    wide = _normal((T, heads * D + 256), g)
    return wide[:, 128:128 + heads * D].view(T, heads, D)


def _lengths(case):
    """(cached tokens with the new ones, new tokens) of every sequence."""
    B, most, new = case["B"], case["len"], case["new"]
    if not case["ragged"]:
        return [most] * B, [new] * B
    rng = random.Random("%d %d %d" % (B, most, new))
    news = [new if new == 1 else rng.randint(1, new) for _ in range(B)]
    lens = [max(n, rng.randint(max(1, most // 16), most)) for n in news]
    lens[0], news[0] = most, new
    return lens, news


def _pages(tokens, page):
    return -(-tokens // page)


def _page_bytes(case):
    n = case["Hkv"] * case["page"]
    return n * case["D"] * 2 if case["cache"] == "fp16" else n * (case["D"] // 2 + 2)


def _plane(case, pages, g):
    n, D = case["Hkv"] * case["page"], case["D"]
    if case["cache"] == "fp16":
        return _normal((pages, n * D), g).view(torch.uint8)
    codes = torch.randint(0, 256, (pages, n * D // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = (torch.rand((pages, n), device="cuda", generator=g) * 0.2 + 0.1).to(torch.float16)
    return torch.cat((codes, scales.view(torch.uint8)), dim=1)


def _prepare_append(case, g):
    lens, news = _lengths(case)
    rows = [_pages(n, case["page"]) for n in lens]
    pages = sum(rows) + 3
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(rows), max(rows) + 1), -1, dtype=torch.int32, device="cuda")
    at, start = 0, [0]
    for i, n in enumerate(rows):
        table[i, :n] = order[at:at + n]
        at += n
        start.append(start[-1] + news[i])
    T, Hq, H, D = start[-1], case["Hq"], case["Hkv"], case["D"]
    q, k, v = torch.split(_rows(T, Hq + 2 * H, D, g), [Hq, H, H], dim=1)
    return {"q": q, "k": k, "v": v, "k_pages": _plane(case, pages, g), "v_pages": _plane(case, pages, g), "table": table,
            "kv_len": _ints(lens), "q_start": _ints(start), "one": max(news) == 1, "T": T}


def _prepare_linear(case, g):
    M, N, K = case["M"], case["N"], case["K"]
    x = _normal((M, K), g)
    x[:, torch.randint(0, K, (max(1, K // 100),), device="cuda", generator=g)] *= 20.0  # outlier channels
    W = torch.empty((N, K), dtype=torch.int8, device="cuda")
    for i in range(0, N, 8192):
        part = _normal((min(8192, N - i), K), g, 32.0, torch.float32)
        W[i:i + 8192] = part.round_().clamp_(-127.0, 127.0).to(torch.int8)
    return {"x": x, "W": W, "s_w": (torch.rand((N,), device="cuda", generator=g) + 0.5) * 6e-4}


def _prepare_sample(case, g):
    B, V = case["B"], case["V"]
    x = _normal((B, V), g, 2.0, torch.float32)
    # a few likely tokens above the bulk
    x += torch.rand((B, V), device="cuda", generator=g).pow_(600).mul_(10.0)
    if case["masked"]:
        x[torch.rand((B, V), device="cuda", generator=g) < 0.3] = -math.inf
        x[:, V - V // 64:] = -math.inf
    one = torch.rand((B, 4), device="cuda", generator=g)
    kind = case["rows"]
    on = torch.tensor([kind in ("top-k",), kind in ("top-p",), False], device="cuda").expand(B, 3)
    if kind == "mixed":  # some rows without a setting, some with several
        on = torch.rand((B, 3), device="cuda", generator=g) < 0.5
    temperature = 0.5 + one[:, 0]
    if kind == "mixed":
        temperature = torch.where(torch.arange(B, device="cuda") % 8 == 3, torch.zeros_like(temperature), temperature)
    return {"logits": x.to(torch.float16) if case["type"] == "fp16" else x, "u": torch.rand((B,), device="cuda", generator=g),
            "temperature": temperature, "top_k": torch.where(on[:, 0], (2.0 * 100.0 ** one[:, 1]).round().to(torch.int32), 0).to(torch.int32),
            "top_p": torch.where(on[:, 1], 0.7 + 0.29 * one[:, 2], 1.0), "min_p": torch.where(on[:, 2], 0.01 + 0.2 * one[:, 3], 0.0)}


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "linear":
        s = _prepare_linear(case, g)
    elif kind == "sample":
        s = _prepare_sample(case, g)
    else:
        freq, mag = _frequencies(case)
        s = {"freq": freq, "mag": mag}
        if kind == "append":
            s |= _prepare_append(case, g)
        else:
            s["x"] = _rows(case["T"], case["heads"], case["D"], g)
            s["positions"] = torch.arange(case["first"], case["first"] + case["T"], dtype=torch.int32, device="cuda")
    return s | {"case": case}


# ---------------------------------------------------------------- one pass


def run(state):
    return (_framework if own else _plain)(state)


def _framework(s):
    import paper_2606_08761_amd as apex4
    c = s["case"]
    if c["kind"] == "rope":
        return apex4.apex4_rope(s["x"], s["positions"], s["freq"], layout=c["layout"], scale=s["mag"])
    if c["kind"] == "linear":
        return apex4.apex4_w8a8_linear(s["x"], s["W"], s["s_w"])
    if c["kind"] == "sample":
        return apex4.apex4_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    start = None if s["one"] else s["q_start"]
    q = apex4.apex4_kv_append_rope(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], c["page"], s["freq"],
                                   layout=c["layout"], scale=s["mag"], q_start=start, cache=c["cache"])
    if c["cache"] == "fp16":
        return q, s["k_pages"].view(torch.float16), s["v_pages"].view(torch.float16)
    return (q, *apex4.apex4_kv_gather(s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["T"], c["Hkv"], c["D"], c["page"],
                                      q_start=start, cache=c["cache"]))


# ---------------------------------------------------------------- the plain forms


def _plain(s):
    return {"rope": _plain_rope, "append": _plain_append, "linear": _plain_linear, "sample": _plain_sample}[s["case"]["kind"]](s)


def _turned(x, positions, s):
    """float32, whatever x is."""
    c = s["case"]
    angle = positions.double()[:, None, None] * s["freq"] * (2 * math.pi)
    cos, sin = (angle.cos() * s["mag"]).float(), (angle.sin() * s["mag"]).float()
    y, rot = x.float(), c["rot"]
    if c["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    return torch.cat((turned, y[..., rot:]), dim=-1)


def _plain_rope(s):
    return _turned(s["x"], s["positions"], s).to(torch.float16)


def _where(s):
    """The sequence of every new token, and its position."""
    start, tok = s["q_start"].long(), torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(start, tok, right=True) - 1
    return seq, s["kv_len"].long()[seq] - start[seq + 1] + tok


def _split(pages, case):
    """Views of a plane: binary16 values [P, Hkv, page, D], or codes [P, Hkv, page, D/2] and scales [P, Hkv, page]."""
    P, H, page, D = pages.shape[0], case["Hkv"], case["page"], case["D"]
    if case["cache"] == "fp16":
        return pages.view(torch.float16).view(P, H, page, D), None
    n = H * page * D // 2
    return pages[:, :n].unflatten(1, (H, page, D // 2)), pages[:, n:].view(torch.float16).unflatten(1, (H, page))


def _stored(x, pages, page, off, case):
    """x [T, Hkv, D] (binary16) into the plane; the values that a 4-bit plane then holds."""
    into, scales = _split(pages, case)
    if scales is None:
        into[page, :, off] = x
        return pages.view(torch.float16)
    v = x.float()
    sc = (v.abs().amax(dim=2) / 7.0).to(torch.float16)
    q = torch.where(sc[..., None] > 0, v / sc.float()[..., None], torch.zeros_like(v)).round().clamp(-8, 7)
    n = q.to(torch.int8).view(torch.uint8) & 15
    into[page, :, off] = n[..., 0::2] | (n[..., 1::2] << 4)
    scales[page, :, off] = sc
    return (q * sc.float()[..., None]).to(torch.float16)


def _plain_append(s):
    c = s["case"]
    seq, pos = _where(s)
    page, off = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    q, k = (_turned(s[x], pos, s).to(torch.float16) for x in ("q", "k"))
    return q, _stored(k, s["k_pages"], page, off, c), _stored(s["v"], s["v_pages"], page, off, c)


def _plain_linear(s):
    x = s["x"].float()
    scale = x.abs().amax(dim=1, keepdim=True) / 127.0
    # quotients next to a half are told apart in 64 bits
    codes = torch.where(scale > 0, x.double() / scale.double(), 0.0).round().clamp(-127.0, 127.0).float()
    return (codes @ s["W"].float().t() * scale * s["s_w"]).to(torch.float16)


def _plain_sample(s):
    """In 64 bits: running sums, and weights next to a border."""
    x, t = s["logits"].double(), s["temperature"].double()[:, None]
    greedy = t <= 0
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, 1.0, t))
    rank = torch.arange(x.shape[1], device="cuda")
    k, p, least = s["top_k"][:, None], s["top_p"].double()[:, None], s["min_p"].double()[:, None]
    inside = torch.where((rank < k) | (k <= 0), w, 0.0)
    before = inside.cumsum(dim=1) - inside
    keep = (before < p * inside.sum(dim=1, keepdim=True)) | (p >= 1.0)
    kept = torch.where((keep & (w >= least)) | (rank == 0), inside, 0.0)
    kept = torch.zeros_like(kept).scatter_(1, order, kept)
    run_ = kept.cumsum(dim=1)
    total = run_[:, -1:]
    token = (run_ <= s["u"].double()[:, None] * total).sum(dim=1, keepdim=True)
    token = torch.where(greedy, order[:, :1], token)
    share = torch.where(greedy, 1.0, kept.gather(1, token) / total)
    return token[:, 0].to(torch.int32), share[:, 0].float()


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    kind = case["kind"]
    if kind == "rope":
        n = case["T"] * case["heads"]
        return {"bytes": 4 * n * case["D"] + 4 * case["T"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    if kind == "append":
        T, H, D = sum(_lengths(case)[1]), case["Hkv"], case["D"]
        token = 2 * H * (2 * D if case["cache"] == "fp16" else D // 2 + 2)
        back = 0 if case["cache"] == "fp16" else token + 4 * H * D
        return {"bytes": T * (4 * case["Hq"] * D + 4 * H * D + token + back), "flops": 3 * T * (case["Hq"] + H) * case["rot"]}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 4 * N + 2 * M * N, "flops": 2 * M * N * K}
    n = case["B"] * case["V"]
    return {"bytes": n * (2 if case["type"] == "fp16" else 4) + 28 * case["B"], "flops": 2 * n}


# ---------------------------------------------------------------- 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_turned(s["x"], s["positions"], s)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "linear":
        return _exact_linear(s)
    return (None, _exact_share(s))


def _exact_turned(x, positions, s):
    """Complex products."""
    c, rot = s["case"], s["case"]["rot"]
    turns = positions.double()[:, None] * s["freq"]
    unit = torch.polar(torch.full_like(turns, s["mag"]), 2 * math.pi * (turns - turns.floor()))[:, None]
    y = x.double()
    out = y.clone()
    if c["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * unit
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * unit
        out[..., 0:rot:2], out[..., 1:rot:2] = z.real, z.imag
    return out


def _exact_append(s):
    c = s["case"]
    lens, news = _lengths(c)
    pos = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(lens, news)])
    q, k = _exact_turned(s["q"], pos, s), _exact_turned(s["k"], pos, s)
    if c["cache"] == "int4":
        return q, _exact_codes(k), _exact_codes(s["v"])
    planes = []
    for x, name in ((k, "k_pages"), (s["v"].double(), "v_pages")):
        plane = s[name].view(torch.float16).double()
        view, at = plane.view(-1, c["Hkv"], c["page"], c["D"]), 0
        for b, (n, m) in enumerate(zip(lens, news)):
            t = torch.arange(n - m, n, device="cuda")
            view[s["table"][b].long()[t // c["page"]], :, t % c["page"]] = x[at:at + m]
            at += m
        planes.append(plane)
    return (q, *planes)


def _exact_codes(x):
    """The cache takes binary16 values and holds them in codes with a binary16 scale."""
    v = x.to(torch.float16).double()
    sc = (v.abs().amax(dim=-1, keepdim=True) / 7.0).to(torch.float16).double()
    return torch.where(sc > 0, (v / sc).round().clamp(-8, 7) * sc, torch.zeros_like(v))


def _exact_linear(s):
    x = s["x"].double()
    scale = (x.abs().amax(dim=1) / 127.0).float().double()  # binary32 by definition
    codes = torch.zeros_like(x)
    some = scale > 0
    codes[some] = (x[some] / scale[some, None]).round().clamp(-127.0, 127.0)
    y = torch.empty((x.shape[0], s["W"].shape[0]), dtype=torch.float64, device="cuda")
    for i in range(0, y.shape[1], 8192):
        y[:, i:i + 8192] = codes @ s["W"][i:i + 8192].double().t().contiguous()
    return y * scale[:, None] * s["s_w"].double()


def _exact_share(s):
    """Row by row: the settings as cuts of the sorted row."""
    x = s["logits"].double()
    out = torch.ones((x.shape[0],), dtype=torch.float64, device="cuda")
    settings = [v.double().tolist() for v in (s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"])]
    for b, (t, k, p, least, u) in enumerate(zip(*settings)):
        if t <= 0:
            continue
        v, at = torch.sort(x[b], descending=True, stable=True)
        w = torch.softmax(v / t, dim=0)
        n = len(w) if k <= 0 else min(int(k), len(w))
        if p < 1:
            so_far = torch.cumsum(w[:n], 0)
            n = min(n, int((so_far < p * so_far[-1]).sum()) + 1)
        n = max(1, min(n, int((w >= least * w[0]).sum())))
        chosen, i = at[:n].sort()
        mass = w[:n][i]
        so_far = torch.cumsum(mass, 0)
        out[b] = mass[(so_far > u * so_far[-1]).to(torch.uint8).argmax()] / so_far[-1]
    return out
