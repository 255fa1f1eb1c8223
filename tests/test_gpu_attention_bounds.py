"""sss_attention without a bound of its requests' tokens but the largest number."""
import pytest
import torch

from test_gpu_attention import BF, FP, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_q", [2 ** 31 - 1, 2 ** 31 - 16, 2 ** 31, 2 ** 32 + 1])
@pytest.mark.parametrize("fresh,kv,hq,hkv,page,dtype", [
    ([40, 70, 1, 100, 33, 9, 64, 20], [300, 70, 90, 333, 33, 9, 1000, 20], 16, 8, 16, BF),
    ([300, 200], [300, 200], 8, 2, 0, FP), ([1, 1], [500, 40], 8, 2, 64, BF), ([20], [4000], 8, 2, 16, BF),
])
def test_every_token_is_written(max_q, fresh, kv, hq, hkv, page, dtype):
    c = make(fresh, kv, hq, hkv, 128, dtype, page, seed=60)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = call(c, max_q=max_q, status=status)
    check(c, got)
    assert int(status) == 0
    assert torch.equal(got, call(c, max_q=sum(fresh)))
