"""Plain 64-bit forms of the paged cache's operators, on the CPU, and inputs for
their tests.  Written from the definitions: loops over sequences and tokens, no
code of the package."""
import math

import numpy as np


def page_bytes(cache, H, D, page):
    return H * page * (2 * D if cache == "fp16" else D // 2 + 2)


def symquant(x):
    """Codes and binary16 scales of rows x [..., D] (one group a row), exact
    quotients: binary16 operands, 64-bit division, ties to even."""
    v = np.asarray(x, np.float64)
    s = (np.abs(v).max(axis=-1) / 7.0).astype(np.float16)
    sd = s.astype(np.float64)[..., None]
    q = np.where(sd > 0, np.divide(v, sd, out=np.zeros_like(v), where=sd > 0), 0.0)
    return np.clip(np.rint(q), -8, 7).astype(np.int8), s


class Plane:
    """One plane on the host: raw bytes, and token access."""

    def __init__(self, cache, pages, H, D, page, raw=None):
        self.cache, self.H, self.D, self.page = cache, H, D, page
        self.raw = np.zeros((pages, page_bytes(cache, H, D, page)), np.uint8) if raw is None else raw
        n = H * page * D // 2
        if cache == "fp16":
            self.f16 = self.raw.view(np.float16).reshape(-1, H, page, D)
        else:
            self.codes = self.raw[:, :n].reshape(-1, H, page, D // 2)
            self.scales = self.raw[:, n:].view(np.float16).reshape(-1, H, page)

    def get(self, page, at):
        """[H, D] float64 of one token."""
        if self.cache == "fp16":
            return self.f16[page, :, at].astype(np.float64)
        c = self.codes[page, :, at].astype(np.int16)
        v = np.empty((self.H, self.D))
        v[:, 0::2] = ((c & 15) ^ 8) - 8
        v[:, 1::2] = ((c >> 4) ^ 8) - 8
        return v * self.scales[page, :, at].astype(np.float64)[:, None]

    def put(self, page, at, x):
        if self.cache == "fp16":
            self.f16[page, :, at] = x
            return
        q, s = symquant(x)
        u = q.view(np.uint8) & 15
        self.codes[page, :, at] = u[:, 0::2] | (u[:, 1::2] << 4)
        self.scales[page, :, at] = s

    def spoil(self, page, at):
        """A token that must not count: NaN (an int4 cache's scales)."""
        if self.cache == "fp16":
            self.f16[page, :, at] = np.nan
        else:
            self.codes[page, :, at] = 0x77
            self.scales[page, :, at] = np.nan


def seen(p, t, window, sinks):
    return 0 <= t <= p and (window == 0 or t > p - window or t < sinks)


def attention(q, K, V, p, window, sinks, scale):
    """One row: q [Hq, D], K and V [tokens, H, D] (64 bits), position p.  Returns
    (out, mean absolute value under the weights, largest value seen) [Hq, D]."""
    Hq, D = q.shape
    H = K.shape[1]
    t = [i for i in range(min(p + 1, K.shape[0])) if seen(p, i, window, sinks)]
    if not t:
        return np.zeros((Hq, D)), np.zeros((Hq, D)), 0.0
    Ks, Vs = K[t], V[t]
    out, mean = np.empty((Hq, D)), np.empty((Hq, D))
    for j in range(Hq):
        h = j // (Hq // H)
        s = Ks[:, h] @ q[j].astype(np.float64) * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        out[j], mean[j] = w @ Vs[:, h], w @ np.abs(Vs[:, h])
    return out, mean, float(np.abs(Vs).max())


def tolerance(out, mean, top, tokens):
    """Bound of a kernel's error against the 64-bit result.  The weights are
    rounded to binary16: 2^-11 of a weight each, so 2^-11 of the weighted mean
    of |v|; as much again for the scores' 32-bit sums (128 products of magnitude
    sum under 2^8: 2^-10 at the very worst, far less in random signs) and the
    exponential; a weight below binary16's normal range errs by 2^-25 of the
    largest one at most, for each token; the output's rounding is 2^-11 of it and
    2^-25 in the subnormal range."""
    return 2.0 ** -10 * mean + 2.0 ** -11 * np.abs(out) + tokens * 2.0 ** -24 * top + 2.0 ** -24


class Case:
    """Sequences in a paged cache, their new tokens last; tokens that no new one
    sees are NaN.  Arrays on the host."""

    def __init__(self, seed, lens, news, Hq, H, D, page, cache, window=0, sinks=0, spare=3, width=None, spoil=True, sd=1.0):
        g = np.random.default_rng(seed)
        self.lens, self.news, self.Hq, self.H, self.D = list(lens), list(news), Hq, H, D
        self.page, self.cache, self.window, self.sinks = page, cache, window, sinks
        rows = [-(-n // page) for n in lens]
        pages = sum(rows) + spare
        order = g.permutation(pages)
        self.width = width or max(max(rows), 1) + 1
        self.table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(rows):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.k, self.v = (Plane(cache, pages, H, D, page) for _ in range(2))
        self.K, self.V = [], []
        for b, n in enumerate(lens):
            for plane, keep in ((self.k, self.K), (self.v, self.V)):
                x = g.standard_normal((n, H, D)).astype(np.float16) * np.float16(sd)
                for t in range(n):
                    plane.put(self.table[b, t // page], t % page, x[t])
                keep.append(np.stack([plane.get(self.table[b, t // page], t % page) for t in range(n)])
                            if n else np.zeros((0, H, D)))
        if spoil:
            self.spoil()
        self.start = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
        self.T = int(self.start[-1])
        self.q = (g.standard_normal((self.T, Hq, D)) * 1.5).astype(np.float16)
        self.scale = 1.0 / math.sqrt(D)

    def spoil(self):
        """Every place of the pool that holds no token that any new one sees."""
        pages = self.k.raw.shape[0]
        used = np.zeros((pages, self.page), bool)
        for b, n in enumerate(self.lens):
            for t in range(n):
                if any(seen(p, t, self.window, self.sinks) for p in (range(n - self.news[b], n) if self.window else (n - 1,))):
                    used[self.table[b, t // self.page], t % self.page] = True
        for p, at in zip(*np.nonzero(~used)):
            self.k.spoil(p, at)
            self.v.spoil(p, at)

    def expected(self):
        """(out, tolerance) [T, Hq, D]."""
        out, tol = np.empty((self.T, self.Hq, self.D)), np.empty((self.T, self.Hq, self.D))
        for b, n in enumerate(self.lens):
            for i in range(self.news[b]):
                r = self.start[b] + i
                p = n - self.news[b] + i
                y, mean, top = attention(self.q[r], self.K[b], self.V[b], p, self.window, self.sinks, self.scale)
                out[r], tol[r] = y, tolerance(y, mean, top, p + 1)
        return out, tol
