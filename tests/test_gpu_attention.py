"""sss_attention against a plain 64-bit form: head layouts, types, lengths from
none to long, pages and packed rows, masks that leave rows empty, what lies where
nothing may be read, strides, streams and refusals of the data.

The tolerance is the bound of attn_plain.attention_bound, derived from the
roundings that the operator makes."""
import math

import numpy as np
import pytest
import torch

import attn_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make(fresh, kv, hq, hkv, dim, dtype, page=0, seed=0, spread=1.0, spare=2, fill=float("nan")):
    """A call's tensors.  page 0: keys packed as the queries.  Slots that hold no
    key of a request are `fill`."""
    g = torch.Generator().manual_seed(seed)
    t = sum(fresh)
    cu = [0]
    for f in fresh:
        cu.append(cu[-1] + f)
    q = (torch.randn((t, hq, dim), generator=g) * spread).to(dtype)
    if page:
        pages = [-(-n // page) for n in kv]
        order = torch.randperm(sum(pages) + spare, generator=g)
        slots = order.numel() * page
        table = torch.full((len(kv), max(pages + [1]) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = order[at:at + n].int()
            at += n
    else:
        slots, table = t, None
    k, v = (torch.full((slots, hkv, dim), fill, dtype=dtype) for _ in range(2))

    def rows(b):
        j = np.arange(kv[b])
        return table[b].numpy()[j // page].astype(np.int64) * page + j % page if page else cu[b] + j

    for b in range(len(kv)):
        r = torch.from_numpy(rows(b))
        k[r] = torch.randn((kv[b], hkv, dim), generator=g).to(dtype)
        v[r] = torch.randn((kv[b], hkv, dim), generator=g).to(dtype)
    return dict(q=q, k=k, v=v, cu=cu, kv=list(kv), table=table, rows=rows, page=page)


def call(c, max_q=None, max_kv=None, scale=None, status=None, kv_len=True, **kw):
    cache = sss.KVCache(c["k"].to(DEV), c["v"].to(DEV), c["page"] or 16)
    fresh = np.diff(c["cu"])
    out = torch.full(c["q"].shape, 7.0, dtype=c["q"].dtype, device=DEV)
    sss.sss_attention(c["q"].to(DEV), cache, torch.tensor(c["cu"], dtype=torch.int32, device=DEV),
                      torch.tensor(c["kv"], dtype=torch.int32, device=DEV) if kv_len else None,
                      int(max(fresh)) if max_q is None else max_q,
                      max(c["kv"]) if max_kv is None else max_kv,
                      block_table=None if c["table"] is None else c["table"].to(DEV),
                      scale=scale, out=out, dev_status=status, **kw)
    torch.cuda.synchronize()
    return out.cpu()


def check(c, got, scale=None):
    dim, dtype = c["q"].shape[2], c["q"].dtype
    want = attn_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"],
                                dim ** -0.5 if scale is None else scale)
    got = got.double().numpy()
    out = want[0]
    fine = np.isfinite(out)
    assert np.array_equal(np.isnan(out), np.isnan(got))
    assert np.array_equal(out[~fine & ~np.isnan(out)], got[~fine & ~np.isnan(out)])
    with np.errstate(all="ignore"):
        bound = attn_plain.attention_bound(*want, dtype, max(c["kv"] + [1]))
    err = np.abs(got - out)
    worst = np.max((err / bound)[fine], initial=0.0)
    assert worst <= 1.0, f"error {worst:.2f} of its bound"


BF, FP = torch.bfloat16, torch.float16

CASES = [
    # fresh, kv, hq, hkv, dim, dtype, page
    # single tokens
    ([1], [1], 1, 1, 64, BF, 16),
    ([1, 1, 1], [1, 16, 17], 8, 2, 128, BF, 16),
    ([1] * 5, [300, 1, 0, 64, 129], 32, 8, 128, BF, 64),
    ([1, 1], [1000, 2500], 16, 2, 128, FP, 32),
    ([1, 1], [700, 33], 40, 1, 64, FP, 128),       # more heads to a group than a tile's rows
    ([1, 1], [513, 255], 7, 1, 128, BF, 256),
    # drafted tokens
    ([2, 5, 3], [2, 77, 400], 8, 2, 128, BF, 16),
    ([5, 5], [900, 1200], 24, 8, 64, BF, 32),
    ([4], [641], 32, 4, 128, FP, 64),
    # prompts, packed
    ([1], [1], 4, 4, 128, BF, 0),
    ([17, 1, 128, 130], [17, 1, 128, 130], 4, 1, 128, BF, 0),
    ([255, 0, 257], [255, 0, 257], 2, 2, 64, BF, 0),
    ([300], [300], 8, 1, 128, FP, 0),
    ([70, 200], [70, 200], 6, 2, 128, BF, 0),      # a group of three
    ([150], [150], 10, 2, 64, FP, 0),              # of five
    ([140], [140], 14, 2, 128, BF, 0),             # of seven
    ([90], [90], 20, 1, 128, BF, 0),               # of twenty
    # chunks of prompts over pages, mixed with single tokens
    ([128, 1, 40], [500, 333, 40], 8, 2, 128, BF, 16),
    ([64], [1087], 8, 8, 128, BF, 64),
    ([33, 200], [290, 201], 16, 2, 64, FP, 128),
    ([100], [613], 4, 1, 128, FP, 256),
    # fewer keys than tokens: the first rows see none
    ([5], [3], 4, 2, 128, BF, 16),
    ([200, 6], [130, 0], 4, 1, 128, BF, 32),
    ([150], [10], 2, 2, 64, FP, 0),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_64_bits(i):
    fresh, kv, hq, hkv, dim, dtype, page = CASES[i]
    c = make(fresh, kv, hq, hkv, dim, dtype, page, seed=100 + i)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check(c, call(c, status=status))
    assert int(status) == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fresh,kv,page", [([1, 1], [700, 90], 16), ([130], [260], 64), ([129], [129], 0)])
def test_sharp_scores(dtype, fresh, kv, page):
    # scores that spread over tens of powers of two: the running maximum rises
    c = make(fresh, kv, 8, 2, 128, dtype, page, seed=7, spread=8.0)
    check(c, call(c))


def test_rising_scores_raise_the_maximum_again_and_again():
    # each block of keys scores higher than the last, by more than the slack
    for fresh, kv, page in (([1], [640], 16), ([128], [640], 64)):
        c = make(fresh, kv, 2, 2, 128, BF, page, seed=8)
        c["q"][:] = 1.0
        for j in range(kv[0]):
            c["k"][c["rows"](0)[j]] = (j // 16) * 0.125
        check(c, call(c, scale=0.7), scale=0.7)


def test_scale():
    for scale in (1e-3, 0.25, 1.0):
        c = make([40, 1], [40, 90], 4, 2, 64, FP, 16, seed=9)
        check(c, call(c, scale=scale), scale=scale)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("fresh,kv,hq,page", [([4], [70], 8, 16), ([100], [100], 4, 0), ([200], [333], 2, 64)])
def test_values_that_no_row_sees_or_some_do(value, fresh, kv, hq, page):
    # a value of one key infinite or NaN: the rows that see the key get it, the
    # others nothing of it; likewise NaN keys (their scores)
    n, m = fresh[0], kv[0]
    for key in (m - 2, m - n + 1, m - 1):
        c = make(fresh, kv, hq, 2, 128, BF, page, seed=key)
        c["v"][c["rows"](0)[key], 1, 5] = value
        c["v"][c["rows"](0)[m - 1], 0, 77] = -value
        check(c, call(c))
    c = make(fresh, kv, hq, 2, 128, BF, page, seed=3)
    c["k"][c["rows"](0)[m - 2], 0, 9] = float("nan")
    check(c, call(c))


def test_infinities_of_both_signs_meet():
    c = make([60], [60], 2, 1, 64, FP, 0, seed=5)
    c["v"][20, 0, 3] = float("inf")
    c["v"][40, 0, 3] = -float("inf")
    c["v"][50, 0, 4] = float("inf")
    check(c, call(c))


@pytest.mark.parametrize("fresh,kv", [([1, 1], [100, 40]), ([150, 20], [150, 90])])
def test_what_lies_past_a_requests_keys_has_no_part(fresh, kv):
    a = make(fresh, kv, 8, 2, 128, BF, 32, seed=11, fill=float("nan"))
    b = make(fresh, kv, 8, 2, 128, BF, 32, seed=11, fill=1000.0)
    assert torch.equal(call(a), call(b))


def test_rows_of_no_request_are_left_alone():
    c = make([3, 2], [30, 20], 4, 2, 64, BF, 16, seed=12)
    c["q"] = torch.cat([c["q"], torch.full((4, 4, 64), float("nan"), dtype=BF)])
    got = call(c)
    assert torch.equal(got[5:], torch.full((4, 4, 64), 7.0, dtype=BF))
    c["q"] = c["q"][:5]
    check(c, got[:5])


@pytest.mark.parametrize("slack", [(3, 100), (200, 5000)])
def test_larger_bounds_than_needed(slack):
    c = make([40, 1], [200, 90], 8, 2, 128, BF, 16, seed=13)
    check(c, call(c, max_q=40 + slack[0], max_kv=200 + slack[1]))


def test_packed_without_kv_len():
    c = make([40, 3, 0, 200], [40, 3, 0, 200], 4, 2, 128, FP, 0, seed=14)
    assert torch.equal(call(c, kv_len=False), call(c))


@pytest.mark.parametrize("page", [0, 64])
def test_strided_queries_and_cache(page):
    # q, k and v columns of one matrix; the result is bit for bit that of dense ones
    c = make([150, 30], [150, 30], 4, 2, 128, BF, page, seed=15)
    dense = call(c)
    slots, t = c["k"].shape[0], c["q"].shape[0]
    kv = torch.randn((slots, 8, 128)).to(BF)
    kv[:, 2:4], kv[:, 5:7] = c["k"], c["v"]
    qs = torch.randn((t, 6, 128)).to(BF)
    qs[:, 1:5] = c["q"]
    kv, qs = kv.to(DEV), qs.to(DEV)
    cache = sss.KVCache(kv[:, 2:4], kv[:, 5:7], page or 16)
    out = sss.sss_attention(qs[:, 1:5], cache, torch.tensor(c["cu"], dtype=torch.int32, device=DEV),
                            torch.tensor(c["kv"], dtype=torch.int32, device=DEV), 150, 150,
                            block_table=None if c["table"] is None else c["table"].to(DEV))
    assert torch.equal(out.cpu(), dense)


def test_other_stream_and_repeats_give_the_same_bits():
    c = make([1, 1, 1], [3000, 700, 60], 16, 2, 128, BF, 16, seed=16)
    first = call(c)
    s = torch.cuda.Stream()
    for _ in range(5):
        assert torch.equal(call(c), first)
        assert torch.equal(call(c, stream=s), first)


def test_in_a_graph():
    c = make([1, 1], [900, 31], 8, 2, 128, BF, 16, seed=17)
    want = call(c)
    cache = sss.KVCache(c["k"].to(DEV), c["v"].to(DEV), 16)
    q, table = c["q"].to(DEV), c["table"].to(DEV)
    cu, kv = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (c["cu"], c["kv"]))
    out = torch.zeros_like(q)
    ws = torch.empty(sss.sss_attention_workspace_bytes(2, 8, cache, 2, 1, 900), dtype=torch.uint8, device=DEV)
    go = lambda: sss.sss_attention(q, cache, cu, kv, 1, 900, block_table=table, out=out,  # noqa: E731
                                   workspace=ws if ws.numel() else None)
    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want)


def test_a_cache_whose_offsets_pass_32_bits():
    # slots x stride x 2 bytes past 2^32, elements past 2^31
    page, hkv, dim = 64, 8, 128
    slots = (2 ** 31 // (hkv * dim) + 4096) // page * page
    k = torch.zeros((slots, hkv, dim), dtype=BF, device=DEV)
    v = torch.zeros((slots, hkv, dim), dtype=BF, device=DEV)
    last = slots // page - 1
    for fresh, kv in (([1], [130]), ([70], [130])):
        c = make(fresh, kv, 16, hkv, dim, BF, page, seed=18, spare=0, fill=0.0)
        pages = [last, 5, last - 3]
        table = torch.tensor([pages], dtype=torch.int32)
        for n, p in enumerate(pages):
            src = c["rows"](0)[n * page:(n + 1) * page]
            k[p * page:p * page + len(src)] = c["k"][src].to(DEV)
            v[p * page:p * page + len(src)] = c["v"][src].to(DEV)
        out = sss.sss_attention(c["q"].to(DEV), sss.KVCache(k, v, page),
                                torch.tensor(c["cu"], dtype=torch.int32, device=DEV),
                                torch.tensor(kv, dtype=torch.int32, device=DEV), fresh[0], 130,
                                block_table=table.to(DEV))
        check(c, out.cpu())


@pytest.mark.parametrize("fresh", [1, 70])
def test_data_out_of_range_raises_the_flag_and_reads_nothing(fresh):
    def flagged(c, **kw):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = call(c, status=status, **kw)
        assert int(status) == sss.FLAG_INDEX
        return out

    base = dict(hq=4, hkv=2, dim=64, dtype=BF, page=16, seed=20)
    # a page that is none: its keys and values read as zeros
    for bad in (-1, 1 << 20, 2 ** 31 - 1):
        c = make([fresh], [100], **base)
        rows = c["rows"](0)[16:32].copy()
        c["table"][0, 1] = bad
        got = flagged(c)
        c["k"][rows], c["v"][rows] = 0, 0
        c["rows"] = lambda b, r=np.concatenate([c["rows"](0)[:16], rows, c["rows"](0)[32:]]): r
        check(c, got)
    # more keys than max_kv: cut there
    c = make([fresh], [100], **base)
    got = flagged(c, max_kv=80)
    c["kv"] = [80]
    check(c, got)
    # a request past the tokens is left out
    c = make([fresh, fresh], [100, 100], **base)
    c["cu"][2] += 5
    got = flagged(c, max_q=fresh + 5)
    assert torch.equal(got[fresh:], torch.full((fresh, 4, 64), 7.0, dtype=BF))


def test_empty_calls_and_python_refusals():
    c = make([1, 1], [10, 20], 4, 2, 64, BF, 16, seed=21)
    cache = sss.KVCache(c["k"].to(DEV), c["v"].to(DEV), 16)
    q, table = c["q"].to(DEV), c["table"].to(DEV)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    kv = torch.tensor([10, 20], dtype=torch.int32, device=DEV)
    assert sss.sss_attention(q[:0], cache, cu[:1], kv[:0], 0, 0).shape == (0, 4, 64)
    bad = [
        (dict(q=q.half()), "bfloat16"), (dict(q=q[..., :32]), "dim"), (dict(q=q.cpu()), "CUDA"),
        (dict(cu=cu.long()), "int32"), (dict(kv=kv[:1]), "elements"), (dict(kv=kv.cpu()), "CUDA"),
        (dict(table=table[:1]), "batch"), (dict(table=table.t()), "batch"),
        (dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), "contiguous"),
        (dict(out=torch.empty((2, 4, 64), dtype=torch.float32, device=DEV)), "bfloat16"),
        (dict(scale=0.0), "SSS_E_ARG"), (dict(scale=float("nan")), "SSS_E_ARG"),
        (dict(q=q[:, :3].contiguous()), "SSS_E_ARG"), (dict(kv=None), "SSS_E_ARG"),
    ]
    for change, what in bad:
        a = dict(q=q, cu=cu, kv=kv, table=table, out=None, scale=None)
        a.update(change)
        with pytest.raises(sss.SssError, match=what):
            sss.sss_attention(a["q"], cache, a["cu"], a["kv"], 1, 20, block_table=a["table"],
                              out=a["out"], scale=a["scale"])


def test_workspace_too_small():
    c = make([20], [4000], 8, 2, 128, BF, 16, seed=22)
    cache = sss.KVCache(c["k"].to(DEV), c["v"].to(DEV), 16)
    need = sss.sss_attention_workspace_bytes(20, 8, cache, 1, 20, 4000)
    assert need > 0  # a chunk of a prompt over 4000 keys is split over CTAs
    with pytest.raises(sss.SssError, match="SSS_E_WORKSPACE"):
        call(c, workspace=torch.empty(need - 16, dtype=torch.uint8, device=DEV))
    check(c, call(c, workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)))


def test_requests_that_run_backwards_raise_the_flag():
    # request 1 ends before it begins; the others are as if it were not there
    c = make([40, 20], [90, 60], 4, 2, 64, BF, 16, seed=23)
    want = call(c)
    bad = dict(c, cu=[0, 60, 40, 60], kv=[60, 60, 60])
    bad["table"] = torch.cat([c["table"][:1], c["table"][1:], c["table"][1:]])
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = call(bad, max_q=60, status=status)
    assert int(status) == sss.FLAG_INDEX
    assert torch.equal(got[40:], want[40:])


def test_a_workspace_of_the_call_is_of_its_stream():
    # what the caller's stream does with its memory meanwhile does not matter
    c = make([20], [6000], 8, 2, 128, BF, 16, seed=24)
    want = call(c)
    cache = sss.KVCache(c["k"].to(DEV), c["v"].to(DEV), 16)
    need = sss.sss_attention_workspace_bytes(20, 8, cache, 1, 20, 6000)
    assert need > 0
    q, table = c["q"].to(DEV), c["table"].to(DEV)
    cu, kv = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (c["cu"], c["kv"]))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(20):
        out = sss.sss_attention(q, cache, cu, kv, 20, 6000, block_table=table, stream=s)
        for _ in range(10):
            torch.empty(need, dtype=torch.uint8, device=DEV).fill_(0xFF)
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want)


def test_a_cache_keeps_its_tensors():
    k = torch.zeros((32, 2, 64), dtype=BF, device=DEV)
    cache = sss.KVCache(k, torch.zeros_like(k))
    with pytest.raises(AttributeError):
        cache.k = torch.zeros_like(k)
    with pytest.raises(AttributeError):
        cache.page_size = 32


@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [
    ([1] * 5, [3000, 1, 65, 0, 700], 64, 2, 128), ([3, 1, 2], [2100, 64, 129], 20, 2, 128),
    ([1] * 3, [1025, 4100, 127], 32, 1, 64), ([2, 2], [2047, 1500], 32, 2, 128),
])
@pytest.mark.parametrize("page", [16, 256])
def test_32_rows_over_many_splits(fresh, kv, hq, hkv, dim, page):
    c = make(fresh, kv, hq, hkv, dim, BF, page, seed=25)
    first = call(c)
    check(c, first)
    assert torch.equal(call(c), first)
