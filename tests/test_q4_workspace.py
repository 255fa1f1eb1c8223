"""sss_attention_q4's workspace: the copy of many rows' keys and values has no more slots than the
bounds of the requests, nor, of several requests, than the cache (no GPU here)."""
import ctypes

import pytest

from paper_2607_08779_gb300 import sss

P = 4096


def size(pages, tokens, heads, width, batch, max_q, max_kv, hkv=8, page=16, dim=128):
    c = sss.KVCacheQ4Desc(P, pages, hkv * (page // 16) * 18 * dim, page, hkv, dim, 0)
    return sss.load().sss_attention_q4_workspace_bytes(tokens, heads, ctypes.byref(c), width, batch, max_q, max_kv)


@pytest.mark.parametrize("batch,pages,max_kv,tokens", [(64, 12500, 131072, 575), (2, 40, 640, 100), (256, 1 << 16, 32768, 3000)])
def test_no_more_than_the_cache(batch, pages, max_kv, tokens):
    copy = 2 * pages * 16 * 8 * 128 * 2
    # besides: fp16 queries and their scales, and what split keys leave (at most one partial result a SM and row tile)
    rest = tokens * 32 * (128 * 2 + 4) + 152 * 256 * (128 + 1) * 4 + 8192
    got = size(pages, tokens, 32, 2 ** 31 - 1, batch, 512, max_kv)
    assert copy <= got <= copy + rest
    # a larger cache: by the requests' bounds, and no more for a table that is wider
    by_requests = 2 * batch * (max_kv // 16) * 16 * 8 * 128 * 2
    assert by_requests > copy
    large = size(1 << 24, tokens, 32, 2 ** 31 - 1, batch, 512, max_kv)
    assert by_requests <= large <= by_requests + rest + batch * (max_kv // 16) * 4
    assert size(pages, tokens, 32, max_kv // 16, batch, 512, max_kv) == got
    assert size(pages, tokens, 32, 2 ** 31 - 1, batch, 1, max_kv) < copy  # single tokens: none


def test_grows_with_the_bounds():
    last = 0
    for max_kv in (16, 100, 640, 1000, 5000, 100000):
        got = size(500, 300, 32, 2 ** 31 - 1, 9, 60, max_kv)
        assert got >= last
        last = got
