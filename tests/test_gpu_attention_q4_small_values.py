"""sss_attention_q4 over values (and keys) that are small for fp16: the error stays relative to
what the cache holds, whose scales are fp16 numbers of 2^-24 and more."""
import math

import numpy as np
import pytest
import torch

import q4_plain
from test_gpu_attention_q4 import BF, FP, call, make

pytestmark = pytest.mark.gpu


def refill(c, name, u, s):
    """The held codes and scales of the call's keys or values."""
    c[name + "c"] = (u, s)
    c[name][0][c["slots"]], c[name][1][c["slots"]] = q4_plain.values(u, s), s


def bound(w, dtype, dim, max_kv, many):
    """As q4_plain's, but with what is lost below fp16's normal range counted as it now is.
    Few rows: p times the scale, in units of 2^-14 of the row's largest p where scales are below 2, is
    rounded by 2^-25 of the unit at most, times a code of 8: 2^-36 a key, over a sum of 1 at
    least; for bf16 p before as well, 2^-39 times the value, which is at most 8 * 2: twice
    that.  Many rows: the copy in fp16 has 11 bits of every value (its least is the scales' own), and p, 2^-8 of
    the row's largest or more, is rounded by 2^-25 of that times the value.  An fp16 output is rounded by
    2^-25 at least."""
    u = q4_plain.UNIT[dtype]
    own = np.maximum(u * np.abs(w["out"]), 2.0 ** -25 if dtype is torch.float16 else 0.0)
    if many:
        h = 2.0 ** -11
        e = 2 * ((dim + 8) * 2.0 ** -23 * (1 + h) + h) * w["reach"] + 2.0 ** -30 * w["coded"]
        e = e[..., None] + max_kv * 2.0 ** -23 + 2.0 ** -20
        return own + (2 * h + h * h + e + e * e) * (1 + u) * w["size"] + max_kv * 2.0 ** -22 * w["most"][..., None]
    h = 2.0 ** -11 if dtype is torch.float16 else 2.0 ** -10 + 2.0 ** -22
    e = 2 * (dim + 16) * 2.0 ** -23 * 24 * w["coded"][..., None] + max_kv * 2.0 ** -22 + 2.0 ** -18
    return own + (h + e) * (1 + u) * w["size"] + max_kv * 2.0 ** -36 * 2


def check(c, got, scale):
    dim, dtype = c["q"].shape[2], c["q"].dtype
    w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], scale)
    most = int(np.diff(c["cu"]).max())
    many = most > 1 and most * (c["q"].shape[1] // c["k"][0].shape[1]) > 64
    err = np.abs(got.double().numpy() - w["out"])
    worst = np.max(err / np.maximum(bound(w, dtype, dim, max(c["kv"]), many), 2.0 ** -149))
    assert worst <= 1.0, f"error {worst:.2f} of its bound"


def flat_but_one(fresh, kv, hq, hkv, dim, dtype, step, gap, seed):
    """Requests whose first key is 2^gap times as heavy as each other one, and holds zeros; the
    others hold values of 1 to 7 steps."""
    c = make(fresh, kv, hq, hkv, dim, dtype, 16, seed=seed)
    rng = np.random.default_rng(seed)
    u, s = c["kc"]
    u[:], s[:] = 8, np.float16(1).view(np.uint16)
    starts = np.cumsum([0] + list(kv[:-1]))
    u[starts, :, 0] = 0  # a code of -8
    refill(c, "k", u, s)
    u, s = c["vc"]
    u[:] = rng.integers(9, 16, u.shape)
    u[starts] = 8
    s[:] = np.float16(step).view(np.uint16)
    refill(c, "v", u, s)
    c["q"][:, :, 0] = -1
    return c, gap * math.log(2) / 8


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("step", [2.0 ** -24, 1.25e-5, 2.0 ** -10])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [([70], [400], 8, 2, 128), ([33, 90], [290, 500], 4, 1, 64)])
def test_small_values_of_many_rows(dtype, step, fresh, kv, hq, hkv, dim):
    c, scale = flat_but_one(fresh, kv, hq, hkv, dim, dtype, step, 2, seed=81)
    check(c, call(c, scale=scale), scale)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("size", [1e-6, 1e-4, 1e-3])
@pytest.mark.parametrize("fresh,kv", [([70, 5], [300, 80])])
def test_small_keys_and_values(dtype, size, fresh, kv):
    # keys and values of a size, queries and scale so that the scores are of order 1
    c = make(fresh, kv, 8, 2, 128, dtype, 16, seed=82, spread=16.0)
    g = np.random.default_rng(82)
    for name in "kv":
        u, s = c[name + "c"]
        new = (size * np.exp(0.5 * g.standard_normal(s.shape)) * g.choice([-1, 1], s.shape)).astype(np.float16)
        refill(c, name, u, new.view(np.uint16))
    scale = 0.01 / size / 16
    check(c, call(c, scale=scale), scale)
