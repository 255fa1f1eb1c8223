"""The bounded wait of the few-row attention's join, made to run out (each CTA expects
16 bytes that nobody stores: all real stores land): the status says so, and the next
call is right."""
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh,kv,hq,dim,dtype", [
    ([1], [2000], 8, 128, BF), ([1] * 5, [3000, 1, 65, 0, 700], 64, 128, BF), ([2, 2], [700, 300], 8, 64, FP),
])
def test_an_expired_join_is_reported_and_leaves_the_gpu_usable(fresh, kv, hq, dim, dtype):
    c = make(fresh, kv, hq, 2, dim, dtype, 16, seed=70)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sss.sss_test_set_stall(sss.TEST_STALL_ATTENTION_ROWS)
    try:
        call(c, status=status)
    finally:
        sss.sss_test_set_stall(0)
    assert int(status) == sss.FLAG_TIMEOUT
    status.zero_()
    check(c, call(c, status=status))
    assert int(status) == 0


def test_the_other_forms_are_not_stalled():
    # keys that one CTA takes whole, and many rows
    for c in (make([1, 1], [60, 30], 8, 2, 128, BF, 16, seed=71), make([40], [90], 8, 2, 128, BF, 16, seed=72)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        sss.sss_test_set_stall(sss.TEST_STALL_ATTENTION_ROWS)
        try:
            got = call(c, status=status)
        finally:
            sss.sss_test_set_stall(0)
        assert int(status) == 0
        check(c, got)
