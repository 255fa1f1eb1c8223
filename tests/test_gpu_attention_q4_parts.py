"""A step that mixes a chunk of a prompt with single tokens as two calls of sss_attention_q4, over
parts of cu_q, the lengths and the table's rows, with the whole step's queries and outputs."""
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention_q4 import BF, DEV, FP, cache_of, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fresh,kv,parts", [
    ([90, 1, 1, 1], [400, 900, 17, 250], [1]), ([1, 1, 70, 1], [33, 300, 70, 1100], [2, 3]), ([1, 0, 2, 128, 50], [5, 9, 700, 128, 333], [3]),
])
def test_parts_of_a_step(dtype, fresh, kv, parts):
    c = make(fresh, kv, 8, 2, 128, dtype, 16, seed=99)
    cache = cache_of(c)
    whole = call(c, cache=cache)
    check(c, whole)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    q, cu, lens, table = c["q"].to(DEV), ints(c["cu"]), ints(kv), c["table"].to(DEV)
    out, status = torch.full(q.shape, 7.0, dtype=dtype, device=DEV), ints([0])
    ends = [0] + parts + [len(fresh)]
    for b0, b1 in zip(ends, ends[1:]):
        before = out.clone()
        sss.sss_attention_q4(q, cache, cu[b0:b1 + 1], lens[b0:b1], max(max(fresh[b0:b1]), 1), max(kv[b0:b1]), table[b0:b1], out=out,
                             dev_status=status)
        at = slice(c["cu"][b0], c["cu"][b1])
        before[at] = out[at]
        assert torch.equal(out, before)  # (the other parts' rows are left alone)
    assert int(status) == 0
    c2 = dict(c)
    # each part within the bounds of its own form, the single tokens' among them
    for b0, b1 in zip(ends, ends[1:]):
        at = slice(c["cu"][b0], c["cu"][b1])
        c2.update(q=c["q"][at], cu=[x - c["cu"][b0] for x in c["cu"][b0:b1 + 1]], kv=kv[b0:b1], rows=lambda b, b0=b0: c["rows"](b0 + b))
        check(c2, out[at].cpu())
