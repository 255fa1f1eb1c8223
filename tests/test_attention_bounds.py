"""Bounds of a request's tokens that are larger than the call: laid out as the call's
tokens are (no GPU here)."""
import ctypes

import pytest

from paper_2607_08779_gb300 import sss
from test_attention_abi import attention, cache

NONE = 2 ** 31 - 1  # "no bound"


@pytest.mark.parametrize("max_q", [NONE, NONE - 1, NONE - 15, NONE - 399, NONE - 4095, 1 << 30, 100000])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,batch,max_kv", [
    (40, 64, 8, 128, 1, 100000), (128, 32, 8, 128, 8, 9000), (300, 32, 8, 128, 2, 3000), (17, 40, 1, 64, 3, 50000),
    (1, 32, 8, 128, 1, 100000), (2, 40, 1, 64, 2, 70000), (1 << 24, 8, 8, 64, 1, 1 << 24),
])
def test_a_bound_above_the_tokens_counts_as_them(max_q, tokens, heads, kv_heads, dim, batch, max_kv):
    if max_q < tokens:
        return
    c = cache(heads=kv_heads, dim=dim, stride=kv_heads * dim, slots=1 << 20)
    size = lambda n: sss.load().sss_attention_workspace_bytes(tokens, heads, ctypes.byref(c), batch, n, max_kv)  # noqa: E731
    assert size(max_q) == size(tokens)


def test_bounds_past_int32_from_python():
    class Cache:  # (what the query reads of a KVCache)
        _ref = ctypes.byref(cache(heads=8, stride=1024))

    size = lambda n: sss.sss_attention_workspace_bytes(64, 32, Cache, 1, n, 8192)  # noqa: E731
    assert size(64) > 0
    for n in (2 ** 31, 2 ** 32 + 1, 2 ** 40):
        assert size(n) == size(64)


@pytest.mark.parametrize("scale,want", [(1e-38, 0), (1e30, 0), (2.2e38, 0), (2.4e38, 1), (2.9e38, 1), (3.4e38, 1)])
def test_scales_whose_product_with_log2_e_is_not_finite(scale, want):
    assert attention(scale=scale) == want
