"""sss_attention_q4 over values (and keys) that are small for fp16: the error stays relative to
what the cache holds, whose scales are fp16 numbers of 2^-24 and more."""
import math

import numpy as np
import pytest
import torch

import q4_plain
from test_gpu_attention_q4 import BF, FP, cache_of, call, make

pytestmark = pytest.mark.gpu


def refill(c, name, u, s):
    """The held codes and scales of the call's keys or values."""
    c[name + "c"] = (u, s)
    c[name][0][c["slots"]], c[name][1][c["slots"]] = q4_plain.values(u, s), s


def bound(w, dtype, dim, max_kv, many):
    """As q4_plain's, but with what is lost below fp16's normal range counted as it now is.
    Few rows: p times the scale, in units of 2^-10 of the row's largest p where scales are below 32, is
    rounded by 2^-25 of the unit at most, times a code of 8: 2^-32 a key, over a sum of 1 at
    least; for bf16 p before as well, by 2^-35 times the value, which is at most 8 times the largest
    scale.  Many rows: the copy in fp16 has 11 bits of every value (its least is the scales' own), and p, 2^-8 of
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
    return own + (h + e) * (1 + u) * w["size"] + max_kv * 2.0 ** -32 * (1 + w["most"][..., None])


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
@pytest.mark.parametrize("step", [2.0 ** -24, 1.25e-5, 2.0 ** -10, 1.0])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim,gap", [
    ([1], [1500], 8, 1, 128, 11), ([1] * 3, [900, 40, 1500], 4, 2, 64, 10), ([3, 1], [700, 1200], 8, 2, 128, 9),
    ([1] * 2, [9000, 12000], 8, 8, 128, 13), ([1] * 40, [250] * 40, 32, 8, 64, 7), ([1] * 2, [1400, 1300], 32, 2, 128, 10),
])
def test_many_keys_of_little_weight(dtype, step, fresh, kv, hq, hkv, dim, gap):
    c, scale = flat_but_one(fresh, kv, hq, hkv, dim, dtype, step, gap, seed=80)
    check(c, call(c, scale=scale), scale)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("step", [2.0 ** -24, 1.25e-5, 2.0 ** -10])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [([70], [400], 8, 2, 128), ([33, 90], [290, 500], 4, 1, 64)])
def test_small_values_of_many_rows(dtype, step, fresh, kv, hq, hkv, dim):
    c, scale = flat_but_one(fresh, kv, hq, hkv, dim, dtype, step, 2, seed=81)
    check(c, call(c, scale=scale), scale)


@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [([70], [4000], 8, 2, 128), ([33, 90], [2900, 700], 4, 1, 64)])
@pytest.mark.parametrize("gap", [20, 27])
def test_keys_of_very_little_weight_in_many_rows(fresh, kv, hq, hkv, dim, gap):
    # bf16 queries: p is lost below 2^-32 of the row's largest (and rounded by 2^-33 of it, times a value of 8 steps)
    c, scale = flat_but_one(fresh, kv, hq, hkv, dim, BF, 1.0, gap, seed=84)
    got = call(c, scale=scale).double().numpy()
    w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], scale)
    limit = bound(w, BF, dim, 0, True) + max(kv) * 2.0 ** -23 * w["size"] + max(kv) * 2.0 ** -30 * w["most"][..., None]
    assert np.max(np.abs(got - w["out"]) / limit) <= 1.0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("size", [1e-6, 1e-4, 1e-3])
@pytest.mark.parametrize("fresh,kv", [([1, 1], [700, 90]), ([2, 1], [1500, 33]), ([70, 5], [300, 80])])
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


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [
    ([1], [1500], 8, 2, 128), ([1, 1], [20, 33], 4, 4, 64), ([4, 3], [300, 200], 8, 2, 128), ([1] * 2, [9000, 300], 8, 8, 128),
    ([1] * 40, [250] * 40, 16, 8, 64),
])
def test_scales_that_grow_and_rows_that_do_not_see_them(dtype, fresh, kv, hq, hkv, dim):
    # each key's scale is at least the ones before it, up to fp16's largest; the last keys' are seen by some rows only
    c = make(fresh, kv, hq, hkv, dim, dtype, 16, seed=83)
    u, s = c["vc"]
    at = 0
    for n in kv:
        new = np.exp2(np.linspace(-24, 15, n)).astype(np.float16)
        s[at:at + n] = new.view(np.uint16)[:, None, None]
        at += n
    refill(c, "v", u, s)
    with np.errstate(all="ignore"):
        w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], dim ** -0.5)
        limit = q4_plain.bound_rows(w, dtype, dim, max(kv))
    cache = cache_of(c)
    got = call(c, cache=cache)
    out = w["out"]
    fits = np.abs(out) <= torch.finfo(dtype).max  # (an fp16 output may not)
    assert np.max((np.abs(got.double().numpy() - out) / limit)[fits]) <= 1.0
    assert torch.equal(got, call(c, cache=cache))
    if max(fresh) > 1:  # the last token's own value is of any scale: the rows before it do not change
        ends = np.cumsum(kv) - 1
        for scale in (2.0 ** -24, 1.0, 3.0, 65504.0):
            s[ends] = np.float16(scale).view(np.uint16)
            refill(c, "v", u, s)
            other = call(c)
            for b in range(len(kv)):
                assert torch.equal(other[c["cu"][b]:c["cu"][b + 1] - 1], got[c["cu"][b]:c["cu"][b + 1] - 1])
