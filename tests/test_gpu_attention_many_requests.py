"""sss_attention of many rows over more requests than a warp has lanes (the search for a
token tile's request takes several turns), groups of heads that leave rows of a tile
empty, and rows that belong to no request."""
import numpy as np
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


def lengths(batch, most, seed):
    """New tokens of each request: single ones, prompts, and none."""
    rng = np.random.default_rng(seed)
    fresh = np.where(rng.random(batch) < 0.5, 1, rng.integers(0, most + 1, batch))
    fresh[rng.integers(0, batch, batch // 8)] = 0
    fresh[batch - 1 - batch // 3] = most
    return fresh


@pytest.mark.parametrize("batch,most,past,hq,hkv,page,dtype", [
    (70, 60, 0, 4, 2, 0, BF),         # packed prompts
    (70, 60, 200, 4, 2, 16, BF),      # chunks and single tokens over pages
    (33, 40, 300, 8, 2, 64, FP), (97, 130, 50, 2, 1, 32, BF), (32, 70, 100, 4, 1, 16, BF), (64, 50, 150, 4, 1, 128, BF),
    (300, 20, 0, 2, 1, 0, FP), (257, 33, 30, 2, 1, 16, BF),
])
def test_many_requests(batch, most, past, hq, hkv, page, dtype):
    fresh = lengths(batch, most, batch)
    held = np.random.default_rng(batch + 1).integers(0, past + 1, batch)
    c = make(fresh.tolist(), (fresh + held).tolist(), hq, hkv, 128, dtype, page, seed=80)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = call(c, status=status)
    check(c, got)
    assert int(status) == 0
    assert torch.equal(call(c), got)


@pytest.mark.parametrize("batch,hq,hkv,dim", [(35, 2, 1, 128), (70, 2, 1, 64), (40, 12, 1, 128)])
def test_many_requests_whose_keys_are_split(batch, hq, hkv, dim):
    fresh = lengths(batch, 20, batch + 2)
    held = np.random.default_rng(batch + 3).integers(0, 400, batch)
    held[[0, 33, batch - 1]] = 3000, 2500, 1999
    c = make(fresh.tolist(), (fresh + held).tolist(), hq, hkv, dim, BF, 16, seed=81)
    cache = sss.KVCache(c["k"].cuda(), c["v"].cuda(), 16)
    assert sss.sss_attention_workspace_bytes(c["q"].shape[0], hq, cache, batch, 20, max(c["kv"])) > 0
    check(c, call(c))


@pytest.mark.parametrize("group", [9, 11, 13, 15])
@pytest.mark.parametrize("fresh,kv,page", [([30, 75], [130, 75], 16), ([100], [100], 0)])
def test_groups_that_leave_rows_empty(group, fresh, kv, page):
    c = make(fresh, kv, 2 * group, 2, 128, BF, page, seed=82)
    check(c, call(c))


@pytest.mark.parametrize("fresh,kv,hq,dim,page", [
    ([40, 130], [200, 130], 8, 128, 16), ([130, 40], [130, 40], 4, 64, 0), ([33], [3000], 8, 128, 64), ([45], [45], 9, 128, 0),
])
def test_rows_of_no_request_are_left_alone(fresh, kv, hq, dim, page):
    # 300 rows past the last request: whole boxes of a tile among them
    hkv = 1 if hq == 9 else 2
    c = make(fresh, kv, hq, hkv, dim, BF, page, seed=83)
    n = sum(fresh)
    more = dict(c, q=torch.cat([c["q"], torch.full((300, hq, dim), float("nan"), dtype=BF)]))
    if not page:  # (the cache has rows for them too)
        more["k"], more["v"] = (torch.cat([c[x], torch.full((300, hkv, dim), float("nan"), dtype=BF)]) for x in "kv")
    got = call(more)
    assert torch.equal(got[n:], torch.full((300, hq, dim), 7.0, dtype=BF))
    check(c, got[:n])
