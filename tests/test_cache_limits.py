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
