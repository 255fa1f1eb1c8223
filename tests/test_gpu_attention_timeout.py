"""The bounded waits of the attention of many rows, made to run out: the status
says so, and the next call is right (the tensor memory was released)."""
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh,kv,page,dtype", [([300], [900], 64, BF), ([40, 200], [40, 200], 0, FP)])
def test_an_expired_wait_is_reported_and_leaves_the_gpu_usable(fresh, kv, page, dtype):
    c = make(fresh, kv, 8, 2, 128, dtype, page, seed=30)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sss.sss_test_set_stall(sss.TEST_STALL_ATTENTION)
    try:
        call(c, status=status)
    finally:
        sss.sss_test_set_stall(0)
    assert int(status) == sss.FLAG_TIMEOUT
    status.zero_()
    check(c, call(c, status=status))
    assert int(status) == 0


def test_single_tokens_have_no_waits_to_stall():
    c = make([1, 1], [700, 30], 8, 2, 128, BF, 16, seed=31)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sss.sss_test_set_stall(sss.TEST_STALL_ATTENTION)
    try:
        got = call(c, status=status)
    finally:
        sss.sss_test_set_stall(0)
    assert int(status) == 0
    check(c, got)


def test_short_items_in_a_row_never_wait_in_vain():
    # requests of one to sixteen key tiles, many to a CTA: whatever role is late, no
    # wait runs out and the bits are the same every time
    fresh = [264, 271, 151, 374, 1200, 164, 36, 32, 342, 26, 129, 128, 257]
    c = make(fresh, fresh, 64, 8, 128, BF, 0, seed=32)
    cache = sss.KVCache(c["k"].cuda(), c["v"].cuda())
    q = c["q"].cuda()
    cu = torch.tensor(c["cu"], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = sss.sss_attention(q, cache, cu, None, 1200, 1200, dev_status=status)
    for _ in range(200):
        out = sss.sss_attention(q, cache, cu, None, 1200, 1200, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.equal(out, first)
