"""The workloads that the speed of the attention step's operators is judged by.

Between a decoder layer's {q, k, v} projection and its o_proj stand three
operators of paper_2607_08779_gb300.sss:

kind     operator            what it is in use
plan     sss_page_plan       once per step of a serving loop: from the requests'
                             lengths the pages they take, the block table, and
                             every token's position and slot
rope     sss_qk_norm_rope    once per layer: the projections' fp32 outputs to the
                             16-bit queries and to the cache's keys and values,
                             heads normalised (or not) and rotated
prompt   sss_attention       once per layer: whole prompts, packed, or chunks of
                             prompts over what the cache holds of them
token    sss_attention       once per layer: single tokens (or a few drafted ones)
                             of each request over the paged cache

A case is a dict of plain values.  Lengths follow from the case alone (`mix` is
the seed that they are spread by), values from the seed.  Head layouts are
Llama3-8B's (32 query heads, 8 of keys and values, of 128), Qwen3-32B's (64 and
8, of 128, with normalised heads) and generic ones in the drawn cases.
"""
import math
import random

import torch

own = False

LLAMA = {"hq": 32, "hkv": 8, "dim": 128}
QWEN = {"hq": 64, "hkv": 8, "dim": 128}


def listed():
    return [
        # one step of a serving loop: sixteen requests decode; and a mixed step of
        # 64 requests, prompts and chunks of them among single tokens
        dict(name="plan_decode_b16", kind="plan", batch=16, page=16, past=8191, fresh=1, spare=0, mix=1),
        dict(name="plan_mixed_b64", kind="plan", batch=64, page=64, past=4096, fresh=2048, spare=37, mix=2),
        # sixteen decoding tokens; the benchmark's prompt of 512 tokens (no norm of
        # the heads); a ragged chunk of 8191 tokens
        dict(name="rope_qwen_b16", kind="rope", tokens=16, norm=True, style="half", rot=128, dtype="bf16", fused=False, page=16, **QWEN),
        dict(name="rope_llama_m512", kind="rope", tokens=512, norm=False, style="half", rot=128, dtype="bf16", fused=False, page=64, **LLAMA),
        dict(name="rope_qwen_m8191", kind="rope", tokens=8191, norm=True, style="half", rot=128, dtype="bf16", fused=False, page=64, **QWEN),
        # the benchmark's prompt; ten prompts of 17 to 2048 tokens packed; a long
        # document; a chunk of 512 tokens after 7680 that the cache holds (fp16)
        dict(name="prompt_llama_m512", kind="prompt", batch=1, low=512, high=512, past=0, page=0, dtype="bf16", mix=3, **LLAMA),
        dict(name="prompt_qwen_ragged_b10", kind="prompt", batch=10, low=17, high=2048, past=0, page=0, dtype="bf16", mix=4, **QWEN),
        dict(name="prompt_llama_m8192", kind="prompt", batch=1, low=8192, high=8192, past=0, page=0, dtype="bf16", mix=5, **LLAMA),
        dict(name="chunk_qwen_m512_past7680", kind="prompt", batch=1, low=512, high=512, past=7680, page=64, dtype="fp16", mix=6, **QWEN),
        # one user; sixteen requests of very different lengths; 64 long ones
        dict(name="token_llama_b1_2k", kind="token", batch=1, low=2047, high=2047, fresh=1, page=16, dtype="bf16", mix=7, **LLAMA),
        dict(name="token_qwen_b16_ragged", kind="token", batch=16, low=130, high=16384, fresh=1, page=64, dtype="bf16", mix=8, **QWEN),
        dict(name="token_llama_b64_16k", kind="token", batch=64, low=12000, high=16384, fresh=1, page=16, dtype="bf16", mix=9, **LLAMA),
    ]


def _log_int(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["plan", "rope", "rope", "prompt", "prompt", "prompt", "token", "token", "token"])
    mix = rng.randrange(1 << 20)
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        return dict(kind=kind, batch=_log_int(rng, 1, 64), page=page, past=_log_int(rng, 1, 8192), fresh=_log_int(rng, 1, 2048),
                    spare=rng.randrange(100), mix=mix)
    hkv = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 8])
    dim = rng.choice([64, 128, 128])
    heads = dict(hq=hkv * group, hkv=hkv, dim=dim, dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if kind == "rope":
        return dict(kind=kind, tokens=_log_int(rng, 1, 8191), norm=rng.random() < 0.5, style=rng.choice(["half", "half", "pairs"]),
                    rot=rng.choice([dim, dim, dim // 2]), fused=rng.random() < 0.3, page=page, **heads)
    if kind == "prompt":
        batch = _log_int(rng, 1, 16)
        high = _log_int(rng, 17, 2048 if batch > 1 else 6000)
        past = 0 if rng.random() < 0.6 else _log_int(rng, 1, 6000)
        # scores of the plain form: at most those of the longest listed prompt
        high = min(high, max(17, int(math.sqrt(past * past / 4 + 2 ** 31 / (batch * hkv * group)) - past / 2)))
        return dict(kind=kind, batch=batch, low=_log_int(rng, 1, high), high=high, past=past,
                    page=page if past or rng.random() < 0.3 else 0, mix=mix, **heads)
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
    if case["kind"] == "plan":
        fresh = [1] * b if case["fresh"] == 1 else _spread(case, 0, 1, case["fresh"], b)
        past = _spread(case, 1, 1, case["past"], b)
        if case["fresh"] > 1:  # some requests are new
            past = [0 if i % 3 == 0 else p for i, p in enumerate(past)]
        return past, fresh
    if case["kind"] == "prompt":
        fresh = _spread(case, 2, case["low"], case["high"], b)
        past = [0] * b if not case["past"] else _spread(case, 3, 1, case["past"], b)
        return past, fresh
    total = _spread(case, 4, case["low"], case["high"], b)
    return [t - case["fresh"] for t in total], [case["fresh"]] * b


def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + 17)
    return g


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _tables(past, total, page, g, spare=0):
    """A block table whose requests hold the pages of `past` tokens, and the
    pages that are free, both in a random order."""
    held = [_cdiv(p, page) for p in past]
    pages = sum(_cdiv(t, page) for t in total) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = max(_cdiv(t, page) for t in total) + 1
    table = torch.full((len(past), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:].contiguous(), pages


def prepare(case, seed):
    from types import SimpleNamespace

    g = _gen(seed)
    s = SimpleNamespace(case=case)
    if case["kind"] == "plan":
        past, fresh = _lengths(case)
        s.past, s.fresh = _int32(past), _int32(fresh)
        s.page = case["page"]
        s.table, s.free, _ = _tables(past, [p + f for p, f in zip(past, fresh)], s.page, g, case["spare"])
        s.tokens = sum(fresh)
        b = case["batch"]
        s.cu_q, s.kv_len, s.used = _int32([0] * (b + 1)), _int32([0] * b), _int32([0])
        s.positions, s.slots = _int32([0] * s.tokens), _int32([0] * s.tokens)
        return s
    hq, hkv, dim, dtype = case["hq"], case["hkv"], case["dim"], DTYPES[case["dtype"]]
    if case["kind"] == "rope":
        t, rot, page = case["tokens"], case["rot"], case["page"]
        # what the projections give: fp32, separate or columns of one matrix
        widths = [hq * dim, hkv * dim, hkv * dim]
        if case["fused"]:
            s.q, s.k, s.v = _normal(g, (t, sum(widths))).split(widths, dim=1)
        else:
            s.q, s.k, s.v = (_normal(g, (t, w)) for w in widths)
        s.wq = 1 + 0.2 * _normal(g, (dim,)) if case["norm"] else None
        s.wk = 1 + 0.2 * _normal(g, (dim,)) if case["norm"] else None
        s.eps, s.half = 1e-6, case["style"] == "half"
        most = 16384
        angle = torch.arange(most, device="cuda", dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot))
        s.cos, s.sin = angle.cos().float(), angle.sin().float()
        start = int(torch.randint(0, most - t, (1,), generator=g, device="cuda"))
        s.positions = torch.arange(start, start + t, device="cuda", dtype=torch.int32)
        pages = _cdiv(t, page) + 3
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        i = torch.arange(t, device="cuda", dtype=torch.int32)
        s.slots = order[(i // page).long()] * page + i % page
        s.page = page
        s.kc, s.vc = (_normal(g, (pages * page, hkv, dim), dtype) for _ in range(2))
        s.q_out = torch.empty((t, hq, dim), dtype=dtype, device="cuda")
        if own:
            from paper_2607_08779_gb300 import sss
            s.cache = sss.KVCache(s.kc, s.vc, page)
            s.rope = sss.Rope(s.cos, s.sin, sss.ROPE_HALF if s.half else sss.ROPE_PAIRS, s.wq, s.wk, s.eps)
        return s
    past, fresh = _lengths(case)
    total = [p + f for p, f in zip(past, fresh)]
    t = sum(fresh)
    # heads of unlike sharpness; the first key of a request draws attention, as a
    # prompt's first token does
    gain = 0.6 + 1.2 * torch.rand((1, hq, 1), generator=g, device="cuda")
    s.q = (_normal(g, (t, hq, dim)) * gain).to(dtype)
    cu = [0]
    for f in fresh:
        cu.append(cu[-1] + f)
    s.cu_q, s.kv_len = _int32(cu), _int32(total)
    s.max_q, s.max_kv = max(fresh), max(total)
    s.page = case["page"]
    if s.page:
        s.table, free, pages = _tables(total, total, s.page, g)
        slots, first = pages * s.page, s.table[:, 0].long() * s.page
    else:  # keys and values packed as the queries are
        s.table, slots, first = None, t, s.cu_q[:-1].long()
    s.kc, s.vc = (_normal(g, (slots, hkv, dim), dtype) for _ in range(2))
    s.kc[first] += 0.25 * s.q[s.cu_q[:-1].long(), ::hq // hkv]
    s.scale = dim ** -0.5
    s.out = torch.empty((t, hq, dim), dtype=dtype, device="cuda")
    if own:
        from paper_2607_08779_gb300 import sss
        s.cache = sss.KVCache(s.kc, s.vc, s.page or 1)
        need = sss.sss_attention_workspace_bytes(t, hq, s.cache, case["batch"], s.max_q, s.max_kv)
        s.workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s.case["kind"]
    if own:
        from paper_2607_08779_gb300 import sss
        if kind == "plan":
            sss.sss_page_plan(s.past, s.fresh, s.page, s.free, s.table, s.cu_q, s.kv_len, s.positions, s.slots, s.used)
            return s.table, s.cu_q, s.kv_len, s.positions, s.slots, s.used
        if kind == "rope":
            sss.sss_qk_norm_rope(s.q, s.k, s.v, s.rope, s.positions, s.cache, slots=s.slots, q_out=s.q_out)
            return s.q_out, s.kc, s.vc
        return sss.sss_attention(s.q, s.cache, s.cu_q, s.kv_len, s.max_q, s.max_kv, block_table=s.table, scale=s.scale,
                                 out=s.out, workspace=s.workspace)
    return {"plan": _plain_plan, "rope": _plain_rope}.get(kind, _plain_attention)(s)


def _plain_plan(s):
    page = s.page
    past, fresh = s.past.long(), s.fresh.long()
    total = past + fresh
    held, pages = (past + page - 1) // page, (total + page - 1) // page
    need = pages - held
    end = need.cumsum(0)
    # the table: column c of request b is a page taken now where held <= c < pages
    c = torch.arange(s.table.shape[1], device="cuda")[None]
    taken = (c >= held[:, None]) & (c < pages[:, None])
    at = (end - need)[:, None] + c - held[:, None]
    free = torch.cat([s.free, s.free.new_full((1,), -1)])  # also where none is free
    s.table.copy_(torch.where(taken, free[at.clamp(0, s.free.numel())], s.table))
    s.cu_q[1:] = fresh.cumsum(0)
    s.kv_len.copy_(total)
    token = torch.arange(s.tokens, device="cuda")
    b = torch.searchsorted(s.cu_q[1:].long(), token, right=True)
    pos = past[b] + token - s.cu_q[b].long()
    s.positions.copy_(pos)
    s.slots.copy_(s.table[b, pos // page] * page + pos % page)
    s.used.copy_(end[-1:])
    return s.table, s.cu_q, s.kv_len, s.positions, s.slots, s.used


def _plain_rope(s):
    c = s.case
    dim, rot = c["dim"], c["rot"]

    def heads(x, w, rotate):
        x = x.reshape(x.shape[0], -1, dim).float()
        if not rotate:
            return x
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s.eps) * w
        cos, sin = s.cos[s.positions.long()][:, None], s.sin[s.positions.long()][:, None]
        r = x[..., :rot]
        if s.half:
            a, b = r[..., :rot // 2], r[..., rot // 2:]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        else:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        return torch.cat([r, x[..., rot:]], dim=-1)

    s.q_out.copy_(heads(s.q, s.wq, True))
    s.kc[s.slots.long()] = heads(s.k, s.wk, True).to(s.kc.dtype)
    s.vc[s.slots.long()] = heads(s.v, None, False).to(s.vc.dtype)
    return s.q_out, s.kc, s.vc


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
    if s.page:
        row = s.table.long()[:, j // s.page] * s.page + j % s.page
    else:
        row = start[:, None] + j
    row = torch.where(inside, row, row[:, :1])
    k, v = (x[row].float().transpose(1, 2) for x in (s.kc, s.vc))  # [b, hkv, max_kv, dim]
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale).view(b, hkv, hq // hkv, s.max_q, s.max_kv)
    seen = j[None, None] <= (kv - n)[:, None, None] + i[None, :, None]
    score.masked_fill_(~(seen & inside[:, None])[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = score.sum(-1).view(b, hkv, -1, 1)
    o = torch.matmul(score.view(b, hkv, -1, s.max_kv), v)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(b, hkv, hq // hkv, s.max_q, dim).permute(0, 3, 1, 2, 4).reshape(b, s.max_q, hq, dim)
    return o[i[None] < n[:, None]].to(s.q.dtype)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    if case["kind"] == "plan":
        past, fresh = _lengths(case)
        taken = sum(_cdiv(p + f, case["page"]) - _cdiv(p, case["page"]) for p, f in zip(past, fresh))
        # lengths; pages taken, read and written; positions and slots
        return {"bytes": 4 * (4 * len(past) + 2 * taken + 2 * sum(fresh)), "flops": 0}
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    if case["kind"] == "rope":
        t, values = case["tokens"], (hq + 2 * hkv) * dim
        return {"bytes": t * (values * 6 + case["rot"] * 4 + 8), "flops": t * (hq + hkv) * dim * (7 if case["norm"] else 3)}
    past, fresh = _lengths(case)
    pairs = sum(f * p + f * (f + 1) // 2 for p, f in zip(past, fresh))
    keys = sum(past) + sum(fresh)
    return {"bytes": 2 * dim * (2 * sum(fresh) * hq + 2 * keys * hkv), "flops": 4 * dim * hq * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "rope": _exact_rope}.get(case["kind"], _exact_attention)(s, case)


def _exact_plan(s, case):
    past, fresh = s.past.tolist(), s.fresh.tolist()
    free, table = s.free.tolist(), s.table.tolist()
    used, cu, positions, slots = 0, [0], [], []
    for b, (p, f) in enumerate(zip(past, fresh)):
        for c in range(_cdiv(p, case["page"]), _cdiv(p + f, case["page"])):
            table[b][c] = free[used]
            used += 1
        for x in range(p, p + f):
            positions.append(x)
            slots.append(table[b][x // case["page"]] * case["page"] + x % case["page"])
        cu.append(cu[-1] + f)
    total = [p + f for p, f in zip(past, fresh)]
    return tuple(_int32(x) for x in (table, cu, total, positions, slots, [used]))


def _exact_rope(s, case):
    t, dim, rot = case["tokens"], case["dim"], case["rot"]
    where = s.positions.long()
    turn = torch.complex(s.cos[where].double(), s.sin[where].double()).unsqueeze(1)

    def one(x, w):
        y = x.double().reshape(t, -1, dim)
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / dim + s.eps).sqrt() * w.double()
        z = y.clone()
        first = slice(0, rot // 2) if s.half else slice(0, rot, 2)
        second = slice(rot // 2, rot) if s.half else slice(1, rot, 2)
        turned = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        z[..., first], z[..., second] = turned.real, turned.imag
        return z

    kc, vc = s.kc.double(), s.vc.double()
    kc[s.slots.long()] = one(s.k, s.wk)
    vc[s.slots.long()] = s.v.double().reshape(t, -1, dim)
    return one(s.q, s.wq), kc, vc


def _exact_attention(s, case):
    past, fresh = _lengths(case)
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    out = torch.zeros((sum(fresh), hq, dim), dtype=torch.float64, device="cuda")
    at = 0
    for b, (p, f) in enumerate(zip(past, fresh)):
        pos = torch.arange(p + f, device="cuda")
        rows = s.table[b, pos // s.page].long() * s.page + pos % s.page if s.page else at + pos
        for h in range(hq):
            k, v = (x[rows, h // (hq // hkv)].double() for x in (s.kc, s.vc))
            for i in range(0, f, 1024):  # a block of queries at a time
                n = min(1024, f - i)
                last = p + i + n
                a = s.q[at + i:at + i + n, h].double() @ k[:last].T * s.scale
                later = pos[:last][None] > p + i + torch.arange(n, device="cuda")[:, None]
                out[at + i:at + i + n, h] = torch.softmax(a.masked_fill(later, -math.inf), dim=-1) @ v[:last]
        at += f
    return out
