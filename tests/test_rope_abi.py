"""Refusals of the rotary position calls (no GPU needed, nothing launched), and the
frequencies against their definitions."""
import math

import pytest

from tests.test_cache_abi import APPEND, BAD_GEOMETRY, L, NULL, P, args  # noqa: F401  (L: the fixture)

ROPE = dict(x=P, x_stride=1024, positions=P, T=5, heads=8, head_dim=128, freq=P, rot=128, layout=0, mag=1.0, out=P, out_stride=1024,
            stream=None)
ROPE_ORDER = "x x_stride positions T heads head_dim freq rot layout mag out out_stride stream".split()
FUSED = dict(q=P, q_stride=1024, heads=8, q_out=P + 16, positions=NULL, freq=P, rot=128, layout=0, mag=1.0, **APPEND)
FUSED_ORDER = ("q q_stride heads q_out k k_stride v v_stride q_start T positions freq rot layout mag k_pages v_pages n_pages table "
               "width kv_len B kv_heads head_dim page cache stream").split()
BAD_ROTARY = [(dict(freq=NULL), -1), (dict(rot=0), -2), (dict(rot=127), -2), (dict(rot=130), -2), (dict(rot=-2), -2), (dict(layout=2), -2),
              (dict(layout=-1), -2), (dict(mag=0.0), -2), (dict(mag=-1.0), -2), (dict(mag=float("nan")), -2), (dict(mag=float("inf")), -2),
              (dict(freq=P + 4), -4)]


@pytest.mark.parametrize("bad,rc", BAD_ROTARY + [
    (dict(x=NULL), -1), (dict(positions=NULL), -1), (dict(out=NULL), -1), (dict(heads=0), -2), (dict(heads=65537), -2),
    (dict(head_dim=0), -2), (dict(head_dim=516, rot=16), -2), (dict(head_dim=520, rot=16), -2), (dict(head_dim=100, rot=16), -2),
    (dict(T=-1), -2), (dict(T=(1 << 24) + 1), -2), (dict(T=1 << 24, heads=9, x_stride=2048, out_stride=2048), -2), (dict(x_stride=1016), -2),
    (dict(x_stride=1028), -2), (dict(out_stride=1016), -2), (dict(out_stride=1026), -2), (dict(out_stride=1032), -2),  # in place: one stride
    (dict(x=P + 8), -4), (dict(out=P + 2), -4), (dict(positions=P + 2), -4)])
def test_rope(L, bad, rc):  # noqa: F811
    assert L.apex4_rope(*args(ROPE_ORDER, ROPE, **bad)) == rc


@pytest.mark.parametrize("bad,rc", BAD_GEOMETRY + BAD_ROTARY + [
    (dict(q=NULL), -1), (dict(q_out=NULL), -1), (dict(k=NULL), -1), (dict(v=NULL), -1), (dict(T=-1), -2), (dict(k_stride=248), -2),
    (dict(v_stride=260), -2), (dict(q_stride=1016), -2), (dict(q_stride=1028), -2), (dict(heads=-1), -2), (dict(heads=65537), -2),
    (dict(q_start=NULL), -2), (dict(q_out=P), -2),  # one token a sequence, but T != B; in place
    (dict(k=P + 8), -4), (dict(v=P + 2), -4), (dict(q=P + 8), -4), (dict(q_out=P + 4), -4), (dict(q_start=P + 2), -4),
    (dict(positions=P + 2), -4), (dict(T=1 << 27), -2)])
def test_append_rope(L, bad, rc):  # noqa: F811
    assert L.apex4_kv_append_rope(*args(FUSED_ORDER, FUSED, **bad)) == rc


def test_without_queries_their_pointers_are_not_asked_for(L):  # noqa: F811
    """What is at fault then is a later check (the page ids' alignment)."""
    assert L.apex4_kv_append_rope(*args(FUSED_ORDER, FUSED, heads=0, q=NULL, q_out=NULL, q_stride=0, table=P + 2)) == -4


@pytest.mark.parametrize("out,out_stride,T", [
    (P + 2032, 2048, 5), (P + 2064, 2048, 5), (P + 16, 2048, 5), (P - 16, 2048, 1), (P + 2032, 2048, 1), (P + 3 * 4096 + 16, 2048, 5),
    (P - 3 * 4096 - 16, 2048, 5), (P + 2048, 1024, 5), (P - 5 * 2048 + 16, 1024, 5)])
def test_outputs_that_overlap(L, out, out_stride, T):  # noqa: F811
    """Rows of 1024 values, those of x 2048 apart: between them is room for out's.  (Without
    an overlap the call would run; that is tested on the device.)"""
    assert L.apex4_rope(*args(ROPE_ORDER, ROPE, x_stride=2048, out=out, out_stride=out_stride, T=T)) == -2
    if out_stride == 1024:  # as q_out, which has no gaps
        far = dict(q=P + (1 << 29), k=P + (1 << 30), v=P + (1 << 31), q_stride=2048, q_out=out, T=T)
        assert L.apex4_kv_append_rope(*args(FUSED_ORDER, FUSED, **{**far, "q": P})) == -2
    for name in ("k", "v"):
        far = dict(q=P + (1 << 29), k=P + (1 << 30), v=P + (1 << 31), q_out=P + 16)
        assert L.apex4_kv_append_rope(*args(FUSED_ORDER, FUSED, **{**far, name: P})) == -2


def test_binding_refuses(L):  # noqa: F811
    import torch

    import paper_2606_08761_amd as pk
    x = torch.zeros((2, 8, 128), dtype=torch.float16)
    with pytest.raises(TypeError):  # host tensors: no CPU path
        pk.apex4_rope(x, torch.zeros(2, dtype=torch.int32), torch.zeros(64, dtype=torch.float64))
    with pytest.raises(TypeError):
        pk.apex4_kv_append_rope(x, x, x, x, x, x, x, 16, x)
    for bad in (dict(rot=7), dict(rot=0), dict(base=1.0), dict(factor=0.0, scaling="linear"), dict(scaling="other"),
                dict(scaling="yarn", low=4.0, high=2.0)):
        with pytest.raises(ValueError):
            pk.apex4_rope_freq(**{"rot": 128, "device": "cpu", **bad})


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_frequencies(rot, base):
    import paper_2606_08761_amd as pk
    plain = [base ** (-2 * j / rot) / (2 * math.pi) for j in range(rot // 2)]

    def near(got, want):
        assert got[0].tolist() == pytest.approx(want, rel=1e-14)
    near(pk.apex4_rope_freq(rot, base, device="cpu"), plain)
    near(pk.apex4_rope_freq(rot, base, "linear", 4.0, device="cpu"), [f / 4 for f in plain])
    f, mag = pk.apex4_rope_freq(rot, base, "yarn", 8.0, 4096, device="cpu")
    assert mag == pytest.approx(0.1 * math.log(8.0) + 1)
    g, one = pk.apex4_rope_freq(rot, base, "bands", 8.0, 4096, device="cpu")
    assert one == 1.0
    for j, p in enumerate(plain):
        turns = p * 4096
        for got, most in ((f, 32.0), (g, 4.0)):
            want = p if turns >= most else p / 8 if turns <= 1.0 else None
            assert want is None and p / 8 <= got[j] <= p or got[j] == pytest.approx(want, rel=1e-12)
    if rot > 2:  # the slowest pair turns factor times slower, the fastest as before
        n = pk.apex4_rope_freq(rot, base, "ntk", 8.0, device="cpu")[0]
        assert n[0] == plain[0] and float(n[-1]) == pytest.approx(plain[-1] / 8, rel=1e-12)


@pytest.mark.parametrize("rot,base,trained,kw,kept", [
    # the ramp's ends: 20.94 and 45.03, so 20 and 46
    (128, 10000.0, 4096, {}, {20: 1, 21: 25 / 26, 30: 16 / 26, 33: 0.5, 45: 1 / 26, 46: 0}),
    (128, 10000.0, 8192, {}, {25: 1, 30: 0.8, 49: 0.04, 50: 0}),                          # 25.76 and 49.84
    (64, 500000.0, 4096, {}, {7: 1, 10: 2 / 3, 15: 1 / 9, 16: 0}),                        # 7.35 and 15.80
    (64, 10000.0, 100, {}, {0: 1, 1: 0.9, 5: 0.5, 10: 0}),                                # -2.43 and 9.61
    (8, 100.0, 16384, dict(high=1000.0, low=0.5), {0: 1, 1: 6 / 7, 3: 4 / 7}),            # 0.83 and 7.43: 7 at most
    (64, 10000.0, 4, {}, {0: 0, 1: 0, 31: 0}),                                            # all turn less than once
    (8, 10000.0, 1 << 40, {}, {0: 1, 1: 1, 3: 1}),                                        # all turn more than 32 times
    (128, 10000.0, 4096, dict(whole_pairs=False),  # from 20.944482 to 45.026881
     {20: 1, 21: 1 - 0.055518 / 24.0824, 33: 1 - 12.055518 / 24.0824, 45: 0.026881 / 24.0824, 46: 0})])
def test_yarn_ramp(rot, base, trained, kw, kept):
    """Pairs between the ramp's ends, worked out by hand: kept shares, the rest 8 times slower."""
    import paper_2606_08761_amd as pk
    f = pk.apex4_rope_freq(rot, base, "yarn", 8.0, trained, device="cpu", **kw)[0]
    for j, keep in kept.items():
        plain = base ** (-2 * j / rot) / (2 * math.pi)
        assert float(f[j]) == pytest.approx(plain * (keep + (1 - keep) / 8), rel=1e-6 if "whole_pairs" in kw else 1e-12), j


def test_bands_ramp():
    """Pairs that turn 2.5 and 1.25 times: (2.5 - 1) / 3 and 0.25 / 3 kept."""
    import paper_2606_08761_amd as pk
    f, mag = pk.apex4_rope_freq(4, 4.0, "bands", 8.0, 2.5 * 2 * math.pi, device="cpu")
    assert mag == 1.0
    for j, keep in ((0, 0.5), (1, 1 / 12)):
        assert float(f[j]) == pytest.approx(0.5 ** j / (2 * math.pi) * (keep + (1 - keep) / 8), rel=1e-12)
