"""Rotary positions: the binding of ``apex4_rope``, and the frequencies that it and
``apex4_kv_append_rope`` take.

    freq, mag = apex4_rope_freq(128)                        # or with a stretched context:
    freq, mag = apex4_rope_freq(128, scaling="yarn", factor=8.0, trained=8192)
    y = apex4_rope(x, positions, freq, scale=mag)           # x [T, heads, head_dim] float16
"""
from __future__ import annotations

import math

from . import _check, _stream, _torch, lib
from .cache import _empty, _freq, _layout, _one_device, _output, _ptr, _rows


def apex4_rope_freq(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: int = 8192,
                    low: float = 1.0, high: float | None = None, device="cuda", whole_pairs: bool = True):
    """(freq, mag): whole turns a position of each of the rot / 2 pairs, float64 [rot / 2],
    and the factor of the turned values.  Unscaled, pair j turns base^(-2 j / rot) radians.

    scaling, for contexts ``factor`` times the trained length:
      "linear"  every pair turns factor times slower (positions interpolated);
      "ntk"     the base grows so that the slowest pair turns factor times slower;
      "yarn"    pairs that turn more than ``high`` (32) times in ``trained`` positions stay,
                those below ``low`` times are slowed, a ramp over the pairs' numbers
                between; mag = 0.1 ln(factor) + 1.  The ramp goes from a whole pair to a
                whole pair, the first number rounded down (0 at least) and the last one up
                (rot - 1 at most), as checkpoints that were trained so expect;
                whole_pairs=False: from and to the very numbers;
      "bands"   the same by the number of turns, from ``high`` (4) down to ``low``."""
    torch = _torch()
    if rot < 2 or rot % 2:
        raise ValueError("rot must be even and at least 2")
    if not (base > 1.0 and factor > 0.0 and trained > 0):
        raise ValueError("base must be above 1, factor and trained above 0")
    n = rot // 2
    j = torch.arange(n, dtype=torch.float64)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2)) if n > 1 else base
    f = base ** (-j / n) / (2 * math.pi)
    mag = 1.0
    if scaling in ("yarn", "bands"):
        high = {"yarn": 32.0, "bands": 4.0}[scaling] if high is None else high
        if not high > low > 0:
            raise ValueError("high must be above low, and low above 0")
        if scaling == "yarn":
            first, last = (n * math.log(trained / (turns * 2 * math.pi)) / math.log(base) for turns in (high, low))
            if whole_pairs:
                first, last = math.floor(first), math.ceil(last)
                if max(first, 0) < min(last, rot - 1):  # else every pair is on one side
                    first, last = max(first, 0), min(last, rot - 1)
            keep = 1.0 - ((j - first) / (last - first)).clamp(0.0, 1.0)
            mag = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
        else:
            keep = ((f * trained - low) / (high - low)).clamp(0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
    elif scaling == "linear":
        f = f / factor
    elif scaling not in ("none", "ntk"):
        raise ValueError("scaling must be 'none', 'linear', 'ntk', 'yarn' or 'bands'")
    return f.to(device), mag


def apex4_rope(x, positions, freq, layout: str = "half", scale: float = 1.0, out=None, stream=None):
    """The first 2 len(freq) values of every head of x [T, heads, head_dim] float16 (rows
    any multiple of 8 apart) turned by positions [T] int32.  out: x itself, or rows like
    x's that do not overlap it (None: made here, without gaps)."""
    torch = _torch()
    xp, xs = _rows(x, "x")
    T, H, D = x.shape
    if positions.dim() != 1 or positions.shape[0] != T:
        raise ValueError("positions must be [T]")
    fp, rot = _freq(freq)
    if out is None:
        out = _empty(x, (T, H, D), torch.float16, stream)
        op, os = out.data_ptr(), H * D
        _one_device(x, positions, freq)
    else:
        op, os = _rows(_output(out, (T, H, D), x, stream), "out")
        _one_device(x, positions, freq, out)
    rc = lib().apex4_rope(xp, xs, _ptr(positions, torch.int32, "positions"), T, H, D, fp, rot, _layout(layout), scale, op, os,
                          _stream(x, stream))
    _check("apex4_rope", rc)
    return out
