"""sss_attention: an infinite value that a row sees reaches its output (infinite, or
NaN where its weight is none), also where the keys are split and the weight of the
split that has it is nothing beside another's."""
import pytest
import torch

from test_gpu_attention import BF, FP, call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fresh,kv,hq", [(1, 2000, 8), (1, 300, 8), (1, 2000, 40), (4, 1500, 8), (40, 3000, 8), (200, 900, 2)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_it_reaches_the_rows_that_see_it(fresh, kv, hq, value, dtype):
    c = make([fresh], [kv], hq, 2, 128, dtype, 64, seed=50)
    rows = c["rows"](0)
    c["q"][:] = c["q"].abs() + 0.5
    c["k"][rows[1:]] = 0.0
    c["k"][rows[0]] = 40.0  # a score of 40 sqrt(128) or so, the others' 0: 2^-600
    want = call(c)
    assert torch.isfinite(want).all()
    for key in (kv - fresh, kv // 2, 1, 70):
        if key > kv - fresh:
            continue
        far = dict(c, v=c["v"].clone())
        far["v"][rows[key], 1, 9] = value
        got = call(far)
        assert not torch.isfinite(got[:, hq // 2:, 9]).any()
        got[:, hq // 2:, 9] = want[:, hq // 2:, 9]
        assert torch.equal(got, want)


@pytest.mark.parametrize("fresh,kv,hq", [(1, 2000, 8), (1, 60, 8), (1, 2000, 40), (4, 1500, 8), (40, 3000, 8), (200, 900, 2)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_it_does_where_all_scores_beside_it_are_minus_infinity(fresh, kv, hq, value):
    c = make([fresh], [kv], hq, 2, 128, BF, 64, seed=51)
    rows = c["rows"](0)
    c["q"][:] = c["q"].abs() + 0.5
    c["k"][rows[1:]] = -float("inf")
    c["k"][rows[0]] = 1.0
    want = call(c)
    assert torch.equal(want, c["v"][rows[0]].repeat_interleave(hq // 2, 0).expand_as(want))
    for key in (kv - fresh, kv // 2, 1, 33):
        far = dict(c, v=c["v"].clone())
        far["v"][rows[key], 1, 9] = value
        got = call(far)
        assert not torch.isfinite(got[:, hq // 2:, 9]).any()
        got[:, hq // 2:, 9] = want[:, hq // 2:, 9]
        assert torch.equal(got, want)
