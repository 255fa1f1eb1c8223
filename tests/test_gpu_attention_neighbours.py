"""sss_attention of many rows: a request's bits are its own.  Its row tiles reach past
its last token (into the next request's queries) and hold rows that no token has
(whatever lay in shared memory): neither may change what its rows give."""
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh,kv,hq,page,dtype", [
    ([300, 64], [300, 64], 8, 0, BF), ([300, 64], [300, 64], 8, 0, FP), ([290, 70, 33], [700, 333, 90], 8, 64, BF),
    ([300, 100], [400, 200], 18, 16, BF), ([280, 130], [280, 130], 2, 0, BF),
])
def test_the_next_requests_queries_do_not_matter(fresh, kv, hq, page, dtype):
    # 300 tokens: the last row tile sees two whole key tiles, and most of its rows are
    # the next request's; sharp queries there raise their maxima again and again
    c = make(fresh, kv, hq, 2, 128, dtype, page, seed=40)
    want = call(c)
    check(c, want)
    for gain in (20.0, -60.0):
        other = dict(c, q=c["q"].clone())
        other["q"][fresh[0]:] *= gain
        assert torch.equal(call(other)[:fresh[0]], want[:fresh[0]])


@pytest.mark.parametrize("group", [3, 5, 6, 7, 9, 12, 20])
def test_what_lay_in_shared_memory_does_not_matter(group):
    # groups whose heads do not fill the 128 rows of a tile; before the call, a call that
    # fills all of them, on every SM
    c = make([300], [700], group, 1, 128, BF, 64, seed=41)
    fill = make([4096], [4096], 8, 2, 128, BF, 0, seed=42)
    cache = sss.KVCache(fill["k"].cuda(), fill["v"].cuda())
    cu = torch.tensor(fill["cu"], dtype=torch.int32, device="cuda")
    got = []
    for gain in (0.0, 20.0, -40.0, 90.0):
        q = (fill["q"] * gain).cuda()
        for _ in range(3):
            sss.sss_attention(q, cache, cu, None, 4096, 4096)
        got.append(call(c))
    check(c, got[0])
    for g in got[1:]:
        assert torch.equal(g, got[0])
