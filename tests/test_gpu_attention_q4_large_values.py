"""sss_attention_q4 of many rows over keys and values that are beyond fp16's range, which its
fp16 copy of them has: they count as 65504, and the status says so."""
import numpy as np
import pytest
import torch

import q4_plain
from paper_2607_08779_gb300 import sss
from test_gpu_attention_q4 import BF, DEV, FP, call, make
from test_gpu_attention_q4_small_values import refill

pytestmark = pytest.mark.gpu


def large(fresh, kv, name, scale, dtype, seed):
    c = make(fresh, kv, 8, 2, 128, dtype, 16, seed=seed)
    u, s = c[name + "c"]
    rng = np.random.default_rng(seed)
    u[:] = rng.integers(0, 16, u.shape)
    u[3:5] = 0  # (codes of -8)
    s[3:5, 1, 2] = np.float16(scale).view(np.uint16)
    refill(c, name, u, s)
    return c


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("scale,over", [(8188.0, False), (-8188.0, False), (8192.0, True), (-9000.0, True), (65504.0, True)])
@pytest.mark.parametrize("fresh,kv", [([70], [300]), ([40, 1], [100, 90])])
def test_beyond_fp16(dtype, name, scale, over, fresh, kv):
    c = large(fresh, kv, name, scale, dtype, seed=90)
    at = 1e-5 if name == "k" else 128 ** -0.5
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = call(c, scale=at, status=status).double().numpy()
    assert int(status) == (sss.FLAG_RANGE if over else 0)
    held = c[name][0].copy()
    c[name] = (np.clip(held, -65504.0, 65504.0), c[name][1])
    assert bool((c[name][0] != held).any()) is over
    w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], at)
    assert np.isfinite(got).all()
    assert np.max(np.abs(got - w["out"]) / q4_plain.bound_many(w, dtype, 128, max(kv))) <= 1.0


def test_keys_that_nobody_sees_say_nothing():
    # slots behind a request's keys, in its last page
    c = make([70], [300], 8, 2, 128, BF, 16, seed=91, fill=0x7B)  # (scales of 61000)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call(c, status=status)
    assert int(status) == 0
    # and those of few rows are taken as they are
    c = large([1], [90], "v", 65504.0, BF, seed=92)
    got = call(c, status=status).double().numpy()
    w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], 128 ** -0.5)
    assert int(status) == 0 and np.abs(w["out"]).max() > 0
    assert np.max(np.abs(got - w["out"]) / q4_plain.bound_rows(w, BF, 128, 90)) <= 1.0
