"""sss_attention_q4 of many rows where its 16-bit copy has the cache's pages: the same bits as with
pages of the requests' own, shared pages and bounds above the lengths among it."""
import numpy as np
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention_q4 import BF, DEV, FP, cache_of, call, check, make

pytestmark = pytest.mark.gpu


def roomy(cache, pages):
    """The same cache with more pages, which nobody holds."""
    big = sss.empty_kv_cache_q4(pages, cache.page_size, cache.blocks.shape[1], cache.blocks.shape[3] // 18)
    big.blocks.fill_(0xFF)
    big.blocks[:cache.blocks.shape[0]] = cache.blocks
    return big


def workspace(c, cache, max_kv):
    fresh = np.diff(c["cu"])
    return sss.sss_attention_q4_workspace_bytes(int(sum(fresh)), c["q"].shape[1], cache, len(c["kv"]), int(max(fresh)), max_kv,
                                                c["table"].shape[1])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim,page", [
    ([70, 1, 33], [300, 90, 33], 8, 2, 128, 16), ([128, 200], [500, 201], 4, 1, 64, 64), ([40, 0, 50], [41, 7, 1200], 16, 2, 128, 256),
])
def test_the_same_bits_as_in_pages_of_their_own(dtype, fresh, kv, hq, hkv, dim, page):
    c = make(fresh, kv, hq, hkv, dim, dtype, page, seed=96)
    wide = torch.full((len(kv), 100), -1, dtype=torch.int32)
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    small = cache_of(c)
    big = roomy(small, 100 * len(kv) + 1)
    for max_kv in (max(kv), 100 * page):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        got = call(c, cache=small, max_kv=max_kv, status=status)
        check(c, got)
        assert torch.equal(got, call(c, cache=big, max_kv=max_kv)) and int(status) == 0
    assert workspace(c, small, 100 * page) < workspace(c, big, 100 * page)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_pages_that_requests_share(dtype):
    # three requests over the same first pages, of unlike lengths; one over nothing but them
    c = make([60, 30, 1, 90], [400, 430, 200, 300], 8, 2, 128, dtype, 16, seed=97)
    small = cache_of(c)
    t = c["table"]
    t[1, :20], t[2, :13], t[3, :19] = t[0, :20], t[0, :13], t[0, :19]
    rows = lambda b: t[b].numpy()[np.arange(c["kv"][b]) // 16].astype(np.int64) * 16 + np.arange(c["kv"][b]) % 16  # noqa: E731
    c["rows"] = rows
    got = call(c, cache=small, max_kv=1000)
    check(c, got)
    assert torch.equal(got, call(c, cache=roomy(small, 1000), max_kv=1000))


def test_pages_that_are_none_and_a_graph():
    c = make([60, 30], [300, 320], 8, 2, 128, BF, 16, seed=98)
    small = cache_of(c)
    bad = c["table"].clone()
    bad[0, 3], bad[1, 2] = -1, 10 ** 6
    for table, flag in ((c["table"], 0), (bad, sss.FLAG_INDEX)):
        c["table"] = table
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        got = call(c, cache=small, max_kv=336, status=status)
        assert int(status) == flag
        status.zero_()
        assert torch.equal(got, call(c, cache=roomy(small, 500), max_kv=336, status=status)) and int(status) == flag
        # a captured call, whose workspace holds anything
        need = workspace(c, small, 336)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        args = (c["q"].to(DEV), small, ints(c["cu"]), ints(c["kv"]), 60, 336, table.to(DEV))
        out, graph = torch.empty_like(args[0]), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sss.sss_attention_q4(*args, out=out, workspace=ws)
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), got)
