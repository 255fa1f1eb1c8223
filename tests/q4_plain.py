"""Plain forms of the 4-bit cache and of the operators on shared pages, and the bounds
of sss_attention_q4's errors, derived from the roundings it makes."""
import numpy as np
import torch

import attn_plain
import oracle
from paper_2607_08779_gb300 import sss

UNIT = attn_plain.UNIT


def quantize(x):
    """Codes c + 8 uint8 and fp16 scales (as uint16 bits) of x [n, heads, dim], by the
    oracle; a scale that overflows is 65504."""
    x = np.ascontiguousarray(x, np.float32)
    n, heads, dim = x.shape
    codes, scales, _, _, flags = oracle.quantize(x.reshape(n * heads, dim), 4, 32, sss.GRID_SIGNED_SYM)
    u = np.stack([codes & 15, codes >> 4], -1).reshape(n, heads, dim)
    s = scales.reshape(n, heads, dim // 32).copy()
    over = (s & 0x7FFF) == 0x7C00
    s[over] -= 1
    return u, s, flags


def values(u, s):
    """float64 values of codes and scale bits."""
    c = u.astype(np.float64) - 8
    return c * np.repeat(s.view(np.float16).astype(np.float64), 32, axis=-1)


def on_grid(x):
    return values(*quantize(x)[:2])


def pack(u, dim, slot_of=None):
    """The code words [n, heads, dim / 8] of codes [n, heads, dim]: by the layout's
    definition, nibble by nibble.  slot_of: the slots' numbers, for values."""
    W = dim // 8
    words = np.zeros(u.shape[:2] + (W,), np.uint32)
    for w in range(W):
        for a in range(4):
            for h in range(2):
                words[..., w] |= u[..., 2 * W * a + W * h + w].astype(np.uint32) << np.uint32(4 * (a + 4 * h))
    if slot_of is not None and dim == 128:
        for i, slot in enumerate(slot_of):
            if slot & 2:
                words[i] = words[i][:, np.arange(W) ^ 8]
    return words


def blocks(k, v, slots, pages, page, heads, dim, fill=0xA5):
    """The cache's bytes with k and v (codes, scale bits) in `slots`, `fill` elsewhere."""
    data = np.full((pages, heads, page // 16, 18 * dim), fill, np.uint8)
    for (u, s), values_too, at in ((k, False, 0), (v, True, 9 * dim)):
        words = pack(u, dim, slots if values_too else None)
        for i, slot in enumerate(slots):
            if slot < 0:
                continue
            j = slot % 16
            for h in range(heads):
                b = data[slot // page, h, slot % page // 16]
                b[at + j * dim // 2:at + (j + 1) * dim // 2] = words[i, h].view(np.uint8)
                b[at + 8 * dim + j * dim // 16:at + 8 * dim + (j + 1) * dim // 16] = s[i, h].view(np.uint8)
    return data


def attention(q, k, v, cu, kv, rows, scale):
    """attn_plain.attention over values k and v (float64 numpy [slots, heads, dim]), and per
    row max_j sum_d |q_d s_jd| scale and sum_d |q_d| scale (for the bounds)."""
    kt, vt = torch.from_numpy(k[0]), torch.from_numpy(v[0])
    out, size, reach, top = attn_plain.attention(q, kt, vt, cu, kv, rows, scale)
    group = q.shape[1] // k[0].shape[1]
    step = np.repeat(np.abs(k[1].view(np.float16).astype(np.float64)), 32, axis=-1)
    vstep = np.abs(v[1].view(np.float16).astype(np.float64)).max(-1)
    coded, most = np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
    qa = q.double().abs().numpy()
    for b in range(len(cu) - 1):
        r = np.asarray(rows(b)[:kv[b]], np.int64)
        for t in range(cu[b], cu[b + 1]):
            for h in range(q.shape[1]):
                if len(r):
                    with np.errstate(all="ignore"):
                        coded[t, h] = (step[r, h // group] @ qa[t, h]).max() * scale
                    most[t, h] = vstep[r, h // group].max()
    return dict(out=out, size=size, reach=reach, coded=coded, most=most, qsum=qa.sum(-1) * scale)


def bound_rows(w, dtype, dim, max_kv):
    """Few rows: scores are dim products of q (exact in fp16 but for what is 2^-28 of its
    row's largest) with codes of at most 15, less 8 times q's sums, added in fp32 (dim + 16
    roundings of 2^-23 of the sizes, which truncation is within), scaled and raised to a power; p times
    the scale is rounded to fp16, by 2^-25 at most below its normal range (times a code, over
    a sum of 1 at least, for every key: 2^-22 each); the output once.  For bf16 p is rounded to
    fp16 before as well: (1 + 2^-11)^2 <= 1 + 2^-10 + 2^-22, and below p's normal range 2^-25
    times the value, of which 2^-25 times its sum is at most 2^-25 of the largest for every key."""
    u = UNIT[dtype]
    h = 2.0 ** -11 if dtype is torch.float16 else 2.0 ** -10 + 2.0 ** -22
    least = 0.0 if dtype is torch.float16 else max_kv * 2.0 ** -25 * 8 * w["most"][..., None]
    e = 2 * (dim + 16) * 2.0 ** -23 * 24 * w["coded"][..., None] + max_kv * 2.0 ** -22 + 2.0 ** -18
    return u * np.abs(w["out"]) + (h + e) * (1 + u) * w["size"] + max_kv * 2.0 ** -22 + least + 2.0 ** -24


def bound_many(w, dtype, dim, max_kv):
    """Many rows: keys and values are rounded to fp16 first (2^-11; below its normal range, of a
    16th of them for bf16, by 2^-25 of what is held), q is exact but for 2^-39 of its row's largest;
    scores of dim products in fp32 (each at most 2^-23 of the products' sizes, taken dim + 8
    times), their scaling and the exponential; p, 2^8 at most, is rounded to fp16 (2^-25 below its normal
    range, for every key, over a sum of 1 at least); sums of max_kv terms that may be
    truncated; the output once."""
    u, h = UNIT[dtype], 2.0 ** -11
    least = 2.0 ** -25 * (1 if dtype is torch.float16 else 16)
    e = 2 * ((dim + 8) * 2.0 ** -23 * (1 + h) + h) * w["reach"] + 2 * least * w["qsum"] + 2.0 ** -30 * w["coded"]
    e = e[..., None] + max_kv * 2.0 ** -23 + 2.0 ** -20
    tiny = 2.0 ** -25 * max_kv * 8 * w["most"][..., None]
    return u * np.abs(w["out"]) + (2 * h + h * h + e + e * e) * (1 + u) * w["size"] + tiny + 2 * least + 2.0 ** -24


def fork(parents, past, page, free, table):
    """(new_table, new_past, src, dst, used) by going through the rows."""
    width = table.shape[1]
    seen, used, rows, lens, src, dst = set(), 0, [], [], [], []
    for p in parents:
        n = past[p] if p >= 0 else 0
        row = [int(x) for x in table[p][:-(-n // page)]] if p >= 0 else []
        a = b = -1
        if n % page and p in seen:
            a, b = row[-1], int(free[used])
            row[-1] = b
            used += 1
        seen.add(p)
        rows.append(row + [-1] * (width - len(row)))
        lens.append(n)
        src.append(a)
        dst.append(b)
    return [np.array(x, np.int64) for x in (rows, lens, src, dst, [used])]


def reclaim(table, past, page, pages, most=None):
    """(free, count) or (free, count, new_table, src, dst, moves)."""
    held = {int(x) for b, row in enumerate(table) for x in row[:-(-past[b] // page)]}
    moves = []
    if most is not None:
        low = iter([x for x in range(pages) if x not in held])
        for a in sorted(held, reverse=True):
            b = next(low, pages)
            if b > a or len(moves) == most:
                break
            moves.append((a, b))
    to = dict(moves)
    held = {to.get(x, x) for x in held}
    free = [x for x in range(pages) if x not in held]
    lists = [np.array(free + [-1] * (pages - len(free))), np.array([len(free)])]
    if most is None:
        return lists
    new = np.array(table)
    for b, row in enumerate(table):
        n = -(-past[b] // page)
        new[b, :n] = [to.get(int(x), int(x)) for x in row[:n]]
    pad = [-1] * (most - len(moves))
    return lists + [new, np.array([a for a, _ in moves] + pad), np.array([b for _, b in moves] + pad),
                    np.array([len(moves)])]
