"""Plain 64-bit forms of the attention step's operators, and the error bounds of
the kernels against them, derived from the roundings they make."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # of the rounding to the type


def page_plan(past, fresh, page, free, table, tokens):
    """(table, cu_q, kv_len, positions, slots, used) by counting."""
    table = np.array(table)
    used, cu, positions, slots = 0, [0], [], []
    for b, (p, f) in enumerate(zip(past, fresh)):
        for c in range(-(-p // page), -(-(p + f) // page)):
            table[b, c] = free[used]
            used += 1
        for x in range(p, p + f):
            positions.append(x)
            slots.append(table[b, x // page] * page + x % page)
        cu.append(cu[-1] + f)
    pad = tokens - len(slots)
    return (table, np.array(cu), np.array(past) + np.array(fresh),
            np.array(positions + [0] * pad), np.array(slots + [-1] * pad), np.array([used]))


def norm_rope(x, w, cos, sin, positions, rot, half, eps, rotate=True):
    """float64 [tokens, heads, dim] of x [tokens, heads, dim], and the sum of the
    sizes of what each value is made of (for the bound)."""
    y = x.astype(np.float64)
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w.astype(np.float64)
    size = np.abs(y)
    if rotate and rot:
        c = cos[positions].astype(np.float64)[:, None]
        s = sin[positions].astype(np.float64)[:, None]
        i = np.arange(rot // 2)
        a, b = (i, i + rot // 2) if half else (2 * i, 2 * i + 1)
        z, size = y.copy(), size.copy()
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., b] * c + y[..., a] * s
        both = np.abs(y[..., a]) + np.abs(y[..., b])
        size[..., a] = size[..., b] = both
        y = z
    return y, size


def norm_rope_bound(y, size, dtype, dim):
    # the sum of dim squares, its root, reciprocal and two products: less than
    # dim + 16 roundings of 2^-24 each; then one rounding to the type
    return UNIT[dtype] * np.abs(y) + (dim + 16) * 2.0 ** -24 * size + 2.0 ** -24


def attention(q, k, v, cu, kv, rows, scale):
    """float64 out [tokens, hq, dim] and its bound's parts.  rows(b): the slots
    of request b's keys.  q, k, v: CPU tensors."""
    hq, dim = q.shape[1:]
    hkv = k.shape[1]
    out = np.zeros(q.shape, np.float64)
    size = np.zeros(q.shape, np.float64)     # sum p |v| / sum p
    reach = np.zeros(q.shape[:2], np.float64)  # max_j sum_d |q_d k_d| scale
    top = np.zeros(q.shape[:2] + (1,), np.float64)
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        r = np.asarray(rows(b)[:kv[b]], np.int64)
        kb, vb = k[r].double().numpy(), v[r].double().numpy()
        for i in range(n):
            lim = max(0, min(kv[b], kv[b] - n + i + 1))
            if lim == 0:
                continue
            t = cu[b] + i
            for h in range(hq):
                g = h // (hq // hkv)
                qi = q[t, h].double().numpy()
                with np.errstate(all="ignore"):
                    s = kb[:lim, g] @ qi * scale
                    p = np.exp(s - s.max())
                    out[t, h] = p @ vb[:lim, g] / p.sum()
                    size[t, h] = p @ np.abs(vb[:lim, g]) / p.sum()
                    reach[t, h] = (np.abs(kb[:lim, g]) @ np.abs(qi)).max() * scale
                    top[t, h] = lim * np.abs(vb[:lim, g]).max()
    return out, size, reach, top


def attention_bound(out, size, reach, top, dtype, max_kv):
    """|result - out| at most: the output's rounding; p rounded to the type; the
    scores' dim products, their scaling and the exponential in fp32 (each at most
    2^-23 of the products' sizes, taken dim + 8 times, in e's exponent); sums of
    max_kv terms that may be truncated; and a p below fp16's normal range is
    rounded to 2^-25, where the row's largest is 1 or more."""
    dim = out.shape[-1]
    u = UNIT[dtype]
    e = 2 * (dim + 8) * 2.0 ** -23 * reach[..., None] + max_kv * 2.0 ** -23 + 2.0 ** -20
    tiny = 2.0 ** -25 * top if dtype is torch.float16 else 0.0
    return u * np.abs(out) + (u + e) * (1 + u) * size + tiny + 2.0 ** -24
