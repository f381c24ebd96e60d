"""Limits that include/apex4.h states for the paged cache's calls, at and past them
(no GPU needed, nothing launched)."""
import pytest

from tests.test_cache_abi import APPEND, APPEND_ORDER, GATHER_ORDER, L, args  # noqa: F401  (L: the fixture)


@pytest.mark.parametrize("T", [(1 << 24) + 1, 1 << 40, 1 << 61, 1 << 62, (1 << 63) - 1])
@pytest.mark.parametrize("kv_heads", [1, 2, 8])
def test_more_tokens_than_a_call_takes(L, T, kv_heads):  # noqa: F811
    """Also where T heads wraps in 64 bits."""
    kw = dict(T=T, kv_heads=kv_heads, k_stride=kv_heads * 128, v_stride=kv_heads * 128)
    assert L.apex4_kv_append(*args(APPEND_ORDER, APPEND, **kw)) == -2
    assert L.apex4_kv_gather(*args(GATHER_ORDER, APPEND, **kw)) == -2


def test_as_many_rows_as_the_header_says(L):  # noqa: F811
    """T heads up to 2^27, inclusive: refused past it, and not at it (what is at fault
    then is a later check: the stride, or the device)."""
    import ctypes
    b = ctypes.c_int64(0)

    def size(T, heads):
        return L.apex4_attn_prefill_workspace_size(T, 4, 8, 4, 64, heads, 1, 128, 16, 0, 0, ctypes.byref(b))
    assert size(1 << 24, 8) != -2 and size(1 << 20, 128) != -2
    assert size(1 << 24, 9) == -2 and size((1 << 20) + 1, 128) == -2
