"""The workloads that the speed of the few-bit cache's and the pages' operators is
judged by.

Next to the attention step on a 16-bit cache (a step's pages, norm and rotation,
attention) stand, in paper_2607_08779_gb300.sss:

kind     operators                         what they are in use
store    sss_kv_store_q4, sss_kv_fetch_q4  once per layer: a step's rotated keys and its
                                           values into the cache in 4 bits; what it holds
                                           of them, read back
token    sss_attention_q4                  once per layer: single tokens (or drafted ones)
                                           of each request over that cache
prompt   sss_attention_q4                  chunks of prompts over what it holds of them
fork     sss_page_fork                     once per step of beams or samples: rows of the
                                           block table from their parents', full pages
                                           shared, the last one copied for all but one
copy     sss_page_copy                     the pages that fork or reclaim want copied, in
                                           all layers' caches
reclaim  sss_page_reclaim                  when requests end or beams are dropped: the free
                                           pages from the block table; with compaction the
                                           pages to move, and the table after it

The cache in 4 bits holds groups of 32 consecutive values x of a head with the
signed scale s = -+ max|x| / 8 whose sign puts the dominant value on the code -8:
c = clip(round(x / s), -8, 7), the value fp16(s) c.

A case is a dict of plain values.  Lengths follow from the case alone (`mix` is
the seed that they are spread by), values from the seed.  Head layouts are
Llama3-8B's (32 query heads, 8 of keys and values, of 128), Qwen3-32B's (64 and
8, of 128) and generic ones in the drawn cases.
"""
import math
import random

import torch

own = False

LLAMA = {"hq": 32, "hkv": 8, "dim": 128}
QWEN = {"hq": 64, "hkv": 8, "dim": 128}


def listed():
    return [
        # a decode step's sixteen tokens; a ragged chunk of 8191 tokens
        dict(name="store_b16", kind="store", tokens=16, hkv=8, dim=128, dtype="fp32", out="fp32", page=16),
        dict(name="store_m8191", kind="store", tokens=8191, hkv=8, dim=128, dtype="bf16", out="bf16", page=64),
        # one user; sixteen requests of very different lengths; 64 long ones
        dict(name="token_llama_b1_2k", kind="token", batch=1, low=2047, high=2047, fresh=1, page=16, dtype="bf16", mix=7, **LLAMA),
        dict(name="token_qwen_b16_ragged", kind="token", batch=16, low=130, high=16384, fresh=1, page=64, dtype="bf16", mix=8, **QWEN),
        dict(name="token_llama_b64_16k", kind="token", batch=64, low=12000, high=16384, fresh=1, page=16, dtype="bf16", mix=9, **LLAMA),
        # a chunk of 512 tokens after 7680 that the cache holds (fp16)
        dict(name="chunk_qwen_m512_past7680", kind="prompt", batch=1, low=512, high=512, past=7680, page=64, dtype="fp16", mix=6, **QWEN),
        # four beams of four requests; 512 samples of 64 long prompts
        dict(name="fork_beams_4x4", kind="fork", batch=16, rows=16, high=2048, page=16, spare=9, mix=10),
        dict(name="fork_samples_512", kind="fork", batch=64, rows=512, high=32768, page=16, spare=40, mix=11),
        # the last pages of those sixteen beams in 32 layers (every fourth keeps its own);
        # the moves of a compaction in a layer of the 16-bit cache
        dict(name="copy_beams_q4_l32", kind="copy", form="q4", layers=32, moves=16, holes=4, pages=64, page=16, hkv=8, dim=128, mix=12),
        dict(name="copy_moves_m500", kind="copy", form="bf16", layers=1, moves=500, holes=0, pages=1500, page=64, hkv=8, dim=128, mix=13),
        # sixteen requests' pages among 4096; 256 requests, beams among them, of a
        # large cache that is to shrink
        dict(name="reclaim_b16", kind="reclaim", batch=16, share=1, high=4096, page=16, fill=0.5, compact=False, most=0, mix=14),
        dict(name="reclaim_compact_b256", kind="reclaim", batch=256, share=4, high=16384, page=16, fill=0.6, compact=True, most=65536, mix=15),
    ]


def _log_int(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["store", "store", "token", "token", "token", "prompt", "prompt", "fork", "copy", "copy", "reclaim", "reclaim"])
    mix = rng.randrange(1 << 20)
    page = rng.choice([16, 32, 64, 128])
    hkv = rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([64, 128, 128])
    if kind == "store":
        return dict(kind=kind, tokens=_log_int(rng, 1, 8191), hkv=hkv, dim=dim, dtype=rng.choice(["fp32", "fp16", "bf16"]),
                    out=rng.choice(["fp32", "fp16", "bf16"]), page=page, mix=mix)
    if kind == "fork":
        batch = _log_int(rng, 1, 64)
        return dict(kind=kind, batch=batch, rows=_log_int(rng, 1, 512), high=_log_int(rng, 1, 32768), page=page,
                    spare=rng.randrange(60), mix=mix)
    if kind == "copy":
        return dict(kind=kind, form=rng.choice(["q4", "bf16", "fp16"]), layers=rng.choice([1, 2, 8, 32]), moves=_log_int(rng, 1, 64),
                    holes=rng.choice([0, 2, 4]), pages=200, page=page, hkv=hkv, dim=dim, mix=mix)
    if kind == "reclaim":
        compact = rng.random() < 0.5
        return dict(kind=kind, batch=_log_int(rng, 1, 256), share=rng.choice([1, 1, 2, 4]), high=_log_int(rng, 1, 16384), page=page,
                    fill=rng.choice([0.3, 0.6, 0.95]), compact=compact, most=_log_int(rng, 1, 65536) if compact else 0, mix=mix)
    group = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 8])
    heads = dict(hq=hkv * group, hkv=hkv, dim=dim, dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if kind == "prompt":
        batch = _log_int(rng, 1, 16)
        high = _log_int(rng, 17, 2048 if batch > 1 else 6000)
        past = 0 if rng.random() < 0.3 else _log_int(rng, 1, 6000)
        # scores of the plain form: at most those of 8192 tokens of 32 heads
        high = min(high, max(17, int(math.sqrt(past * past / 4 + 2 ** 31 / (batch * hkv * group)) - past / 2)))
        return dict(kind=kind, batch=batch, low=_log_int(rng, 1, high), high=high, past=past, page=page, mix=mix, **heads)
    fresh = rng.choice([1, 1, 1, 2, 5])
    batch = _log_int(rng, 1, 64)
    high = _log_int(rng, 16, 32768 if batch <= 16 else 8192)
    return dict(kind=kind, batch=batch, low=min(high, max(fresh, _log_int(rng, 8, high))), high=high, fresh=fresh, page=page, mix=mix, **heads)


# ---------------------------------------------------------------------------
# lengths and inputs
# ---------------------------------------------------------------------------

def _spread(case, salt, lo, hi, n):
    """n lengths from lo to hi over their logarithm; one of them is hi."""
    rng = random.Random(case["mix"] * 31 + salt)
    v = [_log_int(rng, max(1, lo), hi) for _ in range(n)]
    v[rng.randrange(n)] = hi
    return v


def _lengths(case):
    """(past, fresh): per request the tokens that the cache holds already and the
    step's new ones."""
    b = case["batch"]
    if case["kind"] == "prompt":
        fresh = _spread(case, 2, case["low"], case["high"], b)
        past = [0] * b if not case["past"] else _spread(case, 3, max(1, case["past"] // 4), case["past"], b)
        return past, fresh
    total = _spread(case, 4, case["low"], case["high"], b)
    return [t - case["fresh"] for t in total], [case["fresh"]] * b


def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1013 + 29)
    return g


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _heads(g, shape, dtype):
    """Keys or values: dimensions of unlike size, a few of them large."""
    x = torch.randn(shape, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(shape[1:], generator=g, device="cuda"))
    return x.to(dtype)


def _quantize(x):
    """Codes in 0 .. 15, two to a byte, and fp16 scales of x [n, heads, dim]."""
    codes, scales = [], []
    for part in x.split(65536):
        w = part.float().view(*part.shape[:2], -1, 32)
        high, low = w.amax(-1, keepdim=True), w.amin(-1, keepdim=True)
        s = torch.where(high > -low, -high, -low) / 8
        c = (w.double() / torch.where(s == 0, 1.0, s.double())).round().clamp(-8, 7)
        u = (c + 8).to(torch.uint8).flatten(-2)
        codes.append(u[..., 0::2] | u[..., 1::2] << 4)
        scales.append((s + 0.0).squeeze(-1).half())
    return torch.cat(codes), torch.cat(scales)


def _values(codes, scales):
    """The fp32 values that codes [..., dim / 2] and scales [..., dim / 32] stand for."""
    u = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    c = u.float().sub_(8).unflatten(-1, (-1, 32))
    return c.mul_(scales.float().unsqueeze(-1)).flatten(-2)


def _attention_inputs(case, seed):
    """Queries, the block table, and the keys and values before they are put in 4
    bits, in slots."""
    from types import SimpleNamespace

    g = _gen(seed)
    s = SimpleNamespace(case=case)
    hq, hkv, dim, dtype = case["hq"], case["hkv"], case["dim"], DTYPES[case["dtype"]]
    past, fresh = _lengths(case)
    total = [p + f for p, f in zip(past, fresh)]
    t = sum(fresh)
    # heads of unlike sharpness; the first key of a request draws attention, as a
    # prompt's first token does
    gain = 0.6 + 0.9 * torch.rand((1, hq, 1), generator=g, device="cuda")
    s.q = (_normal(g, (t, hq, dim)) * gain).to(dtype)
    cu = [0]
    for f in fresh:
        cu.append(cu[-1] + f)
    s.cu_q, s.kv_len = _int32(cu), _int32(total)
    s.max_q, s.max_kv = max(fresh), max(total)
    s.page = case["page"]
    pages = sum(_cdiv(n, s.page) for n in total)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    s.table = torch.full((len(total), max(_cdiv(n, s.page) for n in total) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(total):
        s.table[b, :_cdiv(n, s.page)] = order[at:at + _cdiv(n, s.page)]
        at += _cdiv(n, s.page)
    s.slots = pages * s.page
    kc = _heads(g, (s.slots, hkv, dim), dtype)
    vc = _heads(g, (s.slots, hkv, dim), dtype)
    kc[s.table[:, 0].long() * s.page] += 0.25 * s.q[s.cu_q[:-1].long(), ::hq // hkv]
    s.scale = dim ** -0.5
    s.out = torch.empty((t, hq, dim), dtype=dtype, device="cuda")
    return s, kc, vc


def _fork_lists(case):
    """(past, parents): beams stay with their request; some parents have many
    children, some none, and a row may be empty."""
    b, rows = case["batch"], case["rows"]
    past = _spread(case, 5, max(1, case["high"] // 8), case["high"], b)
    rng = random.Random(case["mix"] * 31 + 6)
    parents = [min(b - 1, (r * b // rows) // 4 * 4 + rng.randrange(4)) for r in range(rows)]
    if rows > 8:
        parents[rng.randrange(rows)] = -1
    return past, parents


def _reclaim_lists(case):
    """(past, owned): per row the tokens it holds, and the pages that are its own
    (rows come in families of `share` which share all but their last pages)."""
    past = _spread(case, 7, max(1, case["high"] // 8), case["high"], case["batch"])
    share, page = case["share"], case["page"]
    past = [past[b // share * share] for b in range(case["batch"])]
    held = [_cdiv(p, page) for p in past]
    return past, [h if b % share == 0 else min(h, 2) for b, h in enumerate(held)]


def prepare(case, seed):
    from types import SimpleNamespace

    kind = case["kind"]
    if kind in ("token", "prompt"):
        s, kc, vc = _attention_inputs(case, seed)
        if own:
            from paper_2607_08779_gb300 import sss
            s.cache = sss.empty_kv_cache_q4(s.slots // s.page, s.page, case["hkv"], case["dim"])
            sss.sss_kv_store_q4(kc, vc, s.cache)
            need = sss.sss_attention_q4_workspace_bytes(s.q.shape[0], case["hq"], s.cache, case["batch"], s.max_q, s.max_kv)
            s.workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        else:
            s.k, s.v = _quantize(kc), _quantize(vc)
        return s
    g = _gen(seed)
    s = SimpleNamespace(case=case)
    page = s.page = case["page"]
    if kind == "store":
        t, hkv, dim = case["tokens"], case["hkv"], case["dim"]
        s.k, s.v = (_heads(g, (t, hkv, dim), DTYPES[case["dtype"]]) for _ in range(2))
        pages = _cdiv(t, page) + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        i = torch.arange(t, device="cuda", dtype=torch.int32)
        s.slots = order[(i // page).long()] * page + i % page
        s.k_out, s.v_out = (torch.empty((t, hkv, dim), dtype=DTYPES[case["out"]], device="cuda") for _ in range(2))
        if own:
            from paper_2607_08779_gb300 import sss
            s.cache = sss.empty_kv_cache_q4(pages, page, hkv, dim)
        else:
            s.codes = [torch.zeros((pages * page, hkv, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
            s.scales = [torch.zeros((pages * page, hkv, dim // 32), dtype=torch.float16, device="cuda") for _ in range(2)]
    elif kind == "fork":
        past, parents = _fork_lists(case)
        held = [_cdiv(p, page) for p in past]
        order = torch.randperm(sum(held) + case["rows"] + case["spare"], generator=g, device="cuda").to(torch.int32)
        width = max(held) + 1
        s.table = torch.full((case["batch"], width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(held):
            s.table[b, :n] = order[at:at + n]
            at += n
        s.free = order[at:].contiguous()
        s.past, s.parents = _int32(past), _int32(parents)
        rows = case["rows"]
        s.new_table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        s.new_past, s.src, s.dst, s.used = (_int32([0] * n) for n in (rows, rows, rows, 1))
    elif kind == "copy":
        pages, n, hkv, dim = case["pages"], case["moves"], case["hkv"], case["dim"]
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        s.src, s.dst = order[:n].contiguous(), order[n:2 * n].contiguous()
        if case["holes"]:  # entries that ask for no copy
            hole = torch.arange(n, device="cuda") % case["holes"] == case["holes"] - 1
            s.src[hole], s.dst[hole] = -1, -1
        s.layers, s.pages = [], []
        for _ in range(case["layers"]):
            if case["form"] == "q4":
                x = torch.randint(0, 256, (pages, hkv, page // 16, 18 * dim), generator=g, device="cuda", dtype=torch.uint8)
                s.layers.append((x,))
            else:
                s.layers.append(tuple(_normal(g, (pages * page, hkv, dim), DTYPES[case["form"]]) for _ in range(2)))
            s.pages += [x.view(pages, -1) for x in s.layers[-1]]
        if own:
            from paper_2607_08779_gb300 import sss
            s.caches = [sss.KVCacheQ4(*x) if case["form"] == "q4" else sss.KVCache(*x, page) for x in s.layers]
    else:
        past, owned = _reclaim_lists(case)
        pages = max(1, int(sum(owned) / case["fill"]))
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        held = [_cdiv(p, page) for p in past]
        s.table = torch.full((case["batch"], max(held) + 1), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, (h, n) in enumerate(zip(held, owned)):
            if n < h:  # a family shares its first pages
                s.table[b, :h - n] = s.table[b - b % case["share"], :h - n]
            s.table[b, h - n:h] = order[at:at + n]
            at += n
        s.past = _int32(past)
        s.free, s.count = _int32([0] * pages), _int32([0])
        if case["compact"]:
            s.new_table = torch.full_like(s.table, -1)
            s.src, s.dst, s.moves = _int32([0] * case["most"]), _int32([0] * case["most"]), _int32([0])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s.case["kind"]
    if own:
        from paper_2607_08779_gb300 import sss
        if kind == "store":
            sss.sss_kv_store_q4(s.k, s.v, s.cache, s.slots)
            return sss.sss_kv_fetch_q4(s.cache, s.slots, s.k_out, s.v_out)
        if kind == "fork":
            sss.sss_page_fork(s.parents, s.past, s.page, s.free, s.table, s.new_table, s.new_past, s.src, s.dst, s.used)
            return s.new_table, s.new_past, s.src, s.dst, s.used
        if kind == "copy":
            sss.sss_page_copy(s.caches, s.src, s.dst)
            return s.layers
        if kind == "reclaim" and s.case["compact"]:
            sss.sss_page_reclaim(s.table, s.past, s.page, s.free, s.count, s.new_table, s.src, s.dst, s.moves)
            return s.free, s.count, s.new_table, s.src, s.dst, s.moves
        if kind == "reclaim":
            sss.sss_page_reclaim(s.table, s.past, s.page, s.free, s.count)
            return s.free, s.count
        return sss.sss_attention_q4(s.q, s.cache, s.cu_q, s.kv_len, s.max_q, s.max_kv, s.table, scale=s.scale,
                                    out=s.out, workspace=s.workspace)
    return {"store": _plain_store, "fork": _plain_fork, "copy": _plain_copy, "reclaim": _plain_reclaim}.get(kind, _plain_attention)(s)


def _plain_store(s):
    slots = s.slots.long()
    for x, codes, scales, out in zip((s.k, s.v), s.codes, s.scales, (s.k_out, s.v_out)):
        codes[slots], scales[slots] = _quantize(x)
        out.copy_(_values(codes[slots], scales[slots]))
    return s.k_out, s.v_out


def _plain_attention(s):
    hq, hkv, dim = s.case["hq"], s.case["hkv"], s.case["dim"]
    b = s.cu_q.numel() - 1
    start, n, kv = s.cu_q[:-1].long(), s.cu_q.diff().long(), s.kv_len.long()
    i = torch.arange(s.max_q, device="cuda")
    j = torch.arange(s.max_kv, device="cuda")
    # every request padded to the longest: queries [b, hkv, group * max_q, dim]
    token = (start[:, None] + i).clamp(max=s.q.shape[0] - 1)
    q = s.q[token].float().view(b, s.max_q, hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, dim)
    inside = j[None] < kv[:, None]
    row = s.table.long()[:, j // s.page] * s.page + j % s.page
    row = torch.where(inside, row, row[:, :1])
    k, v = (_values(codes[row], scales[row]).transpose(1, 2) for codes, scales in (s.k, s.v))  # [b, hkv, max_kv, dim]
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale).view(b, hkv, hq // hkv, s.max_q, s.max_kv)
    seen = j[None, None] <= (kv - n)[:, None, None] + i[None, :, None]
    score.masked_fill_(~(seen & inside[:, None])[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = score.sum(-1).view(b, hkv, -1, 1)
    o = torch.matmul(score.view(b, hkv, -1, s.max_kv), v)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(b, hkv, hq // hkv, s.max_q, dim).permute(0, 3, 1, 2, 4).reshape(b, s.max_q, hq, dim)
    return o[i[None] < n[:, None]].to(s.q.dtype)


def _plain_fork(s):
    page, width = s.page, s.table.shape[1]
    p = s.parents.long()
    real = p >= 0
    at = p.clamp(min=0)
    past = torch.where(real, s.past[at], 0)
    r = torch.arange(p.numel(), device="cuda")
    # the first row of each parent
    first = torch.full((s.past.numel(),), p.numel(), dtype=torch.int64, device="cuda")
    first = first.scatter_reduce(0, at, torch.where(real, r, p.numel()), "amin")[at]
    copied = real & (past % page > 0) & (first != r)
    new = s.free[(copied.long().cumsum(0) - 1).clamp(min=0)]
    c = torch.arange(width, device="cuda")
    held = (past + page - 1) // page
    t = torch.where((c < held[:, None]) & real[:, None], s.table[at], -1)
    last = copied[:, None] & (c == held[:, None] - 1)
    s.src.copy_(torch.where(copied, t.gather(1, (held.long() - 1).clamp(min=0)[:, None]).squeeze(1), -1))
    s.dst.copy_(torch.where(copied, new, -1))
    s.new_table.copy_(torch.where(last, new[:, None], t))
    s.new_past.copy_(past)
    s.used.copy_(copied.sum().view(1))
    return s.new_table, s.new_past, s.src, s.dst, s.used


def _plain_copy(s):
    src, dst = s.src.long(), s.dst.long()
    # an entry that asks for nothing repeats one that does
    some = (src >= 0).int().argmax()
    src, dst = torch.where(src < 0, src[some], src), torch.where(dst < 0, dst[some], dst)
    for x in s.pages:
        x[dst] = x[src]
    return s.layers


def _plain_reclaim(s):
    page, pages = s.page, s.free.numel()
    held = (s.past + page - 1) // page
    c = torch.arange(s.table.shape[1], device="cuda")
    inside = c < held[:, None]
    mark = torch.zeros(pages + 1, dtype=torch.int64, device="cuda")
    mark[torch.where(inside, s.table, pages).long()] = 1
    mark = mark[:pages]
    x = torch.arange(pages, device="cuda")
    below = mark.cumsum(0) - mark  # held pages before each page
    m = mark.sum()
    if s.case["compact"]:
        # the i-th lowest free page takes the i-th highest held one, while that is higher
        most = s.src.numel()
        k = ((mark == 0) & (x < m)).sum().clamp(max=most)
        s.moves.copy_(k.view(1))
        lists = torch.full((2, max(most, pages) + 1), -1, dtype=torch.int32, device="cuda")
        to, frm = x - below, m - 1 - below
        moved = (mark == 1) & (frm < k)
        taken = (mark == 0) & (to < k)
        spare = lists.shape[1] - 1
        lists[0].scatter_(0, torch.where(moved, frm, spare), x.int())
        lists[1].scatter_(0, torch.where(taken, to, spare), x.int())
        s.src.copy_(lists[0, :most])
        s.dst.copy_(lists[1, :most])
        where = torch.where(moved, lists[1][frm.clamp(0, spare)].long(), x)
        t = s.table.long().clamp(min=0)
        s.new_table.copy_(torch.where(inside, where[t].int(), s.new_table))
        mark = torch.where(moved, 0, torch.where(taken, 1, mark))
        below = mark.cumsum(0) - mark
    free = torch.full((pages + 1,), -1, dtype=torch.int32, device="cuda")
    free.scatter_(0, torch.where(mark == 0, x - below, pages), x.int())
    s.free.copy_(free[:pages])
    s.free.masked_fill_(x >= pages - m, -1)
    s.count.copy_((pages - m).view(1))
    if s.case["compact"]:
        return s.free, s.count, s.new_table, s.src, s.dst, s.moves
    return s.free, s.count


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "store":
        n, size = case["tokens"] * case["hkv"] * case["dim"] * 2, {"fp32": 4, "bf16": 2, "fp16": 2}
        # values read; codes and scales written, and read; values written; slots twice
        return {"bytes": int(n * (size[case["dtype"]] + 2 * 9 / 16 + size[case["out"]])) + 8 * case["tokens"], "flops": 4 * n}
    if kind == "copy":
        entries = case["moves"] - (case["moves"] // case["holes"] if case["holes"] else 0)
        slot = case["hkv"] * case["dim"] * 2 * (9 / 16 if case["form"] == "q4" else 2)
        return {"bytes": int(2 * entries * case["layers"] * case["page"] * slot) + 8 * case["moves"], "flops": 0}
    if kind == "fork":
        past, parents = _fork_lists(case)
        width = _cdiv(max(past), case["page"]) + 1
        used = {p for p in parents if p >= 0}
        held = sum(_cdiv(past[p], case["page"]) for p in used)
        return {"bytes": 4 * (held + len(parents) * (width + 4) + len(past) + len(parents)), "flops": 0}
    if kind == "reclaim":
        past, owned = _reclaim_lists(case)
        held, pages = sum(_cdiv(p, case["page"]) for p in past), max(1, int(sum(owned) / case["fill"]))
        more = held + 2 * case["most"] if case["compact"] else 0
        return {"bytes": 4 * (len(past) + held + pages + more), "flops": 0}
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    past, fresh = _lengths(case)
    pairs = sum(f * p + f * (f + 1) // 2 for p, f in zip(past, fresh))
    keys = sum(past) + sum(fresh)
    return {"bytes": 4 * dim * sum(fresh) * hq + 2 * keys * hkv * dim * 9 // 16, "flops": 4 * dim * hq * pairs}


def exact(case, seed):
    kind = case["kind"]
    if kind in ("token", "prompt"):
        return _exact_attention(case, seed)
    s = prepare(case, seed)
    if kind == "store":
        return tuple(_on_grid(x) for x in (s.k, s.v))
    if kind == "copy":
        src, dst = s.src.tolist(), s.dst.tolist()
        for layer in s.layers:
            for x in layer:
                y = x.view(case["pages"], -1)
                for a, b in zip(src, dst):
                    if a >= 0:
                        y[b] = y[a]
        return s.layers
    return _exact_fork(s, case) if kind == "fork" else _exact_reclaim(s, case)


def _on_grid(x):
    """The values that the cache holds of x [n, heads, dim], in 64 bits."""
    parts = []
    for part in x.split(32768):
        w = part.double().reshape(*part.shape[:-1], -1, 32)
        dominant = w.abs().amax(-1, keepdim=True)
        up = (w == dominant).any(-1, keepdim=True) & ~(w == -dominant).any(-1, keepdim=True)
        step = dominant * torch.where(up, -0.125, 0.125)
        y = torch.where(dominant > 0, w / step, 0.0)
        low = y.floor()
        c = low + ((y - low > 0.5) | ((y - low == 0.5) & (low % 2 != 0)))
        parts.append((c.clamp(max=7) * step.half().double()).flatten(-2))
    return torch.cat(parts)


def _exact_attention(case, seed):
    s, kc, vc = _attention_inputs(case, seed)
    past, fresh = _lengths(case)
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    out = torch.zeros((sum(fresh), hq, dim), dtype=torch.float64, device="cuda")
    at = 0
    for b, (p, f) in enumerate(zip(past, fresh)):
        pos = torch.arange(p + f, device="cuda")
        rows = s.table[b, pos // s.page].long() * s.page + pos % s.page
        kb, vb = (_on_grid(x[rows]) for x in (kc, vc))
        for h in range(hq):
            k, v = kb[:, h // (hq // hkv)], vb[:, h // (hq // hkv)]
            for i in range(0, f, 1024):  # a block of queries at a time
                n = min(1024, f - i)
                last = p + i + n
                a = s.q[at + i:at + i + n, h].double() @ k[:last].T * s.scale
                later = pos[:last][None] > p + i + torch.arange(n, device="cuda")[:, None]
                out[at + i:at + i + n, h] = torch.softmax(a.masked_fill(later, -math.inf), dim=-1) @ v[:last]
        at += f
    return out


def _exact_fork(s, case):
    past, parents, free, table = s.past.tolist(), s.parents.tolist(), s.free.tolist(), s.table.tolist()
    page, width = case["page"], s.table.shape[1]
    seen, used, rows, lens, src, dst = set(), 0, [], [], [], []
    for p in parents:
        n = past[p] if p >= 0 else 0
        row = table[p][:_cdiv(n, page)] if p >= 0 else []
        src.append(-1)
        dst.append(-1)
        if n % page and p in seen:
            src[-1], dst[-1] = row[-1], free[used]
            row = row[:-1] + [free[used]]
            used += 1
        seen.add(p)
        rows.append(row + [-1] * (width - len(row)))
        lens.append(n)
    return tuple(_int32(x) for x in (rows, lens, src, dst, [used]))


def _exact_reclaim(s, case):
    past, table, pages, page = s.past.tolist(), s.table.tolist(), s.free.numel(), case["page"]
    held = {x for b, row in enumerate(table) for x in row[:_cdiv(past[b], page)]}
    moves = []
    if case["compact"]:
        low = (x for x in range(pages) if x not in held)
        for a in sorted(held, reverse=True):
            b = next(low, pages)
            if b > a or len(moves) == case["most"]:
                break
            moves.append((a, b))
        to = dict(moves)
        held = {to.get(x, x) for x in held}
    free = [x for x in range(pages) if x not in held]
    lists = _int32(free + [-1] * (pages - len(free))), _int32([len(free)])
    if not case["compact"]:
        return lists
    new = s.new_table.tolist()
    for b, row in enumerate(table):
        n = _cdiv(past[b], page)
        new[b][:n] = [to.get(x, x) for x in row[:n]]
    pad = [-1] * (case["most"] - len(moves))
    return lists + tuple(_int32(x) for x in (new, [a for a, _ in moves] + pad, [b for _, b in moves] + pad, [len(moves)]))
