"""The bounded wait of sss_attention_q4's join, made to run out (each CTA expects 16 bytes
that nobody stores: all real stores land): the status says so, and the next call is right."""
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention_q4 import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh,kv,hq,dim,dtype", [
    ([1], [2000], 8, 128, BF), ([1, 1], [1500, 60], 64, 128, FP), ([2, 2], [700, 300], 8, 64, FP),
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
