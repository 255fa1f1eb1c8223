"""The attention step's calls with the compiled part of the binding and without: the
same kernels, the same bits."""
import pytest
import torch

import test_gpu_page_plan
import test_gpu_qk_norm_rope
from paper_2607_08779_gb300 import sss
from test_gpu_attention import BF, call, make

pytestmark = pytest.mark.gpu


def test_the_same_bits_either_way(monkeypatch):
    past, fresh = [10, 0, 40], [30, 5, 1]
    table, free = test_gpu_page_plan.setup(past, fresh, 16)
    c = test_gpu_qk_norm_rope.make(20, 8, 2, 128, seed=3)
    out = torch.empty((20, 8, 128), dtype=BF, device="cuda")
    a = make([70, 1], [900, 40], 8, 2, 128, BF, 16, seed=4)

    def step():
        plan, status = test_gpu_page_plan.call(past, fresh, 16, free, table, 36)
        rope = [t.clone() for t in test_gpu_qk_norm_rope.call(c, q_out=out)]
        return [torch.from_numpy(p) for p in plan] + rope + [call(a)], status

    assert sss._binding() is not sss._NoBinding  # (it is there on this machine)
    with_it, s1 = step()
    monkeypatch.setattr(sss, "_fast", sss._NoBinding)
    without, s2 = step()
    assert s1 == s2 == 0
    for x, y in zip(with_it, without):
        assert torch.equal(x, y)
