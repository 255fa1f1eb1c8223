"""A step with more new tokens than its buffers have rows: what is left of it is a step
of its own, with the keys that its tokens have."""
import numpy as np
import pytest

import attn_plain
from paper_2607_08779_gb300 import sss
from test_gpu_page_plan import call, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("past,fresh,tokens,left", [
    ([0, 0], [3, 4], 5, [3, 2]), ([20, 7, 100], [30, 40, 2], 33, [30, 3, 0]), ([5], [600], 257, [257]),
    ([1] * 300, [2] * 300, 401, [2] * 200 + [1] + [0] * 99), ([0, 9], [10, 3], 0, [0, 0]),
])
def test_what_is_left_is_a_step_of_its_own(past, fresh, tokens, left):
    table, free = setup(past, fresh, 16)
    got, status = call(past, fresh, 16, free, table, tokens)
    want = attn_plain.page_plan(past, left, 16, free, table, tokens)
    assert status == sss.FLAG_INDEX
    for i in (1, 2, 3):  # cu_q, kv_len, positions
        assert np.array_equal(got[i], want[i])
