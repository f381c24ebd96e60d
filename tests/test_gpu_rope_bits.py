"""The bits of rotary positions.  Every rounding of the turned values is part of what
include/apex4.h says: sines times mag to binary32, two products and their sum in binary32,
then binary16.  So a value has one right answer, and so has the 4-bit code that it becomes
on its way into a cache, next to a code's border too."""
import numpy as np
import pytest

from tests.test_gpu_attn import dev

pytestmark = pytest.mark.gpu
F32 = np.float32


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def pairs(x, n, layout):
    i, j = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    return i, j, x[..., i], x[..., j]


def bounds(x, positions, freq, layout, mag):
    """The lowest and the highest binary16 result.  Position times frequency and what is left
    past whole turns are the kernel's numbers (one rounding, then none); 2 pi times it is off by
    2^-52, either library's sine and cosine by less than 2^-52: together below 2^-50 mag,
    which the result may be from binary64's before it is rounded to binary32."""
    n = len(freq)
    t = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    angle = 2 * np.pi * (t - np.rint(t))
    c, s, off = np.cos(angle) * mag, np.sin(angle) * mag, 2.0 ** -50 * mag
    i, j, a, b = pairs(x.astype(F32), n, layout)
    low, high = x.copy(), x.copy()
    for place, first in ((i, True), (j, False)):
        found = []
        for dc in (-off, off):
            for ds in (-off, off):
                cf, sf = (c + dc).astype(F32), (s + ds).astype(F32)
                found.append((a * cf - b * sf if first else b * cf + a * sf).astype(np.float16))
        low[..., place], high[..., place] = np.minimum.reduce(found), np.maximum.reduce(found)
    return low, high


def in_64_bits(x, positions, freq, layout, mag):
    t = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    angle = 2 * np.pi * (t - np.rint(t))
    i, j, a, b = pairs(x.astype(np.float64), len(freq), layout)
    y = x.copy()
    y[..., i], y[..., j] = a * (np.cos(angle) * mag) - b * (np.sin(angle) * mag), b * (np.cos(angle) * mag) + a * (np.sin(angle) * mag)
    return y


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,rot", [(1500, 8, 128, 128), (2001, 5, 64, 64), (1000, 5, 128, 64), (900, 7, 96, 6), (700, 3, 72, 72), (500, 3, 256, 256)])
def test_bits(pk, layout, T, H, D, rot):
    """Some hundred of these values would be others with an fma in place of a product and a
    sum, with binary64 up to the end, or with mag rounded to binary32."""
    g = np.random.default_rng(T)
    x = g.standard_normal((T, H, D)).astype(np.float16)
    positions = np.arange(T, dtype=np.int32) * 3
    freq, mag = pk.apex4_rope_freq(rot, scaling="yarn", factor=8.0)
    low, high = bounds(x, positions, freq.cpu().numpy(), layout, mag)
    assert (low != high).sum() <= 1e-5 * x.size
    y = pk.apex4_rope(dev(x), dev(positions), freq, layout=layout, scale=mag).cpu().numpy()
    assert ((low <= y) & (y <= high)).all(), int(((low > y) | (y > high)).sum())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(128, 64), (128, 12), (64, 32)])
def test_codes_next_to_a_border(pk, layout, D, rot):
    """Keys whose turned value is one binary16 number in binary32 and its neighbour in 64
    bits, beside a value that is not turned and gives a scale with a code's border between the
    two: each row has a code that is another in 64 bits."""
    import torch
    g = np.random.default_rng(D + rot)
    T, page = 60000, 16
    freq, mag = pk.apex4_rope_freq(rot, scaling="yarn", factor=8.0)
    f = freq.cpu().numpy()
    x = g.standard_normal((T, 1, D)).astype(np.float16)
    x[..., rot:] = 0
    positions = g.integers(0, 9000, T).astype(np.int32)
    low, high = bounds(x, positions, f, layout, mag)
    other = in_64_bits(x, positions, f, layout, mag)
    at = [(t, e) for t, _, e in np.argwhere((low == high) & (other != low)) if (low[t] == high[t]).all()]
    rows = []
    for t, e in at:
        lo, hi = sorted((abs(float(low[t, 0, e])), abs(float(other[t, 0, e]))))
        most = np.abs(low[t]).max()
        for k in range(7):
            s = np.float16(hi / (k + 0.5))  # the largest scale with the border at hi or below
            if float(s) * (k + 0.5) > hi:
                s = np.nextafter(s, np.float16(0))
            top = np.float16(7 * float(s))
            parted = s > 0 and np.rint(lo / float(s)) != np.rint(hi / float(s))  # a tie goes to the even code
            if parted and top >= most and np.float16(F32(top) / F32(7)) == s:
                x[t, 0, rot] = low[t, 0, rot] = top
                rows.append(t)
                break
    rows = np.unique(rows)
    assert len(rows) >= 20
    k, want = x[rows], low[rows].astype(np.float64)
    scale = (np.abs(want).max(axis=-1, keepdims=True).astype(F32) / F32(7)).astype(np.float16).astype(np.float64)
    want = (np.clip(np.rint(want / scale), -8, 7) * scale).astype(np.float16)
    n = len(rows)
    planes = [torch.zeros((-(-n // page), page * (D // 2 + 2)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = dev(np.arange(-(-n // page), dtype=np.int32)[None])
    lens, start = dev(np.array([n], np.int32)), dev(np.array([0, n], np.int32))
    pk.apex4_kv_append_rope(None, dev(k), dev(np.ones_like(k)), *planes, table, lens, page, freq, layout=layout, scale=mag, q_start=start,
                            positions=dev(positions[rows]), cache="int4")
    got = pk.apex4_kv_gather(*planes, table, lens, n, 1, D, page, q_start=start, cache="int4")[0].cpu().numpy()
    assert np.array_equal(got, want), int((got != want).any(axis=(1, 2)).sum())
