"""sss_attention_q4 against a plain 64-bit form over the values that the cache holds: head
layouts, types, lengths from none to long, pages, masks that leave rows empty, what
lies where nothing may be read, strides, streams and refusals of the data.

The tolerances are the bounds of q4_plain, derived from the roundings that the operator
makes."""
import numpy as np
import pytest
import torch

import q4_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, FP = torch.bfloat16, torch.float16


def make(fresh, kv, hq, hkv, dim, dtype, page=16, seed=0, spread=1.0, spare=2, fill=0xFF):
    """A call's tensors.  Bytes that hold no key of a request are `fill` (0xFF: scales that
    are NaN)."""
    g = torch.Generator().manual_seed(seed)
    t, cu = sum(fresh), [0]
    for f in fresh:
        cu.append(cu[-1] + f)
    q = (torch.randn((t, hq, dim), generator=g) * spread).to(dtype)
    pages = [-(-n // page) for n in kv]
    order = torch.randperm(sum(pages) + spare, generator=g)
    table = torch.full((len(kv), max(pages + [1]) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n].int()
        at += n

    def rows(b):
        j = np.arange(kv[b])
        return table[b].numpy()[j // page].astype(np.int64) * page + j % page

    slots = np.concatenate([rows(b) for b in range(len(kv))] + [np.zeros(0, np.int64)])
    x = [torch.randn((len(slots), hkv, dim), generator=g) * torch.exp(0.7 * torch.randn((1, hkv, dim), generator=g))
         for _ in range(2)]
    c = dict(q=q, cu=cu, kv=list(kv), table=table, rows=rows, page=page, pages=order.numel(), slots=slots, fill=fill)
    for name, y in zip("kv", x):
        u, s, _ = q4_plain.quantize(y.numpy())
        val, sc = np.zeros((order.numel() * page, hkv, dim)), np.zeros((order.numel() * page, hkv, dim // 32), np.uint16)
        val[slots], sc[slots] = q4_plain.values(u, s), s
        c[name] = (val, sc)
        c[name + "c"] = (u, s)
    return c


def cache_of(c):
    hkv, dim = c["k"][0].shape[1:]
    data = q4_plain.blocks(c["kc"], c["vc"], c["slots"].tolist(), c["pages"], c["page"], hkv, dim, fill=c["fill"])
    return sss.KVCacheQ4(torch.from_numpy(data).to(DEV))


def call(c, max_q=None, max_kv=None, scale=None, status=None, cache=None, **kw):
    fresh = np.diff(c["cu"])
    out = torch.full(c["q"].shape, 7.0, dtype=c["q"].dtype, device=DEV)
    sss.sss_attention_q4(c["q"].to(DEV), cache or cache_of(c), torch.tensor(c["cu"], dtype=torch.int32, device=DEV),
                         torch.tensor(c["kv"], dtype=torch.int32, device=DEV), int(max(fresh)) if max_q is None else max_q,
                         max(c["kv"]) if max_kv is None else max_kv, c["table"].to(DEV), scale=scale, out=out,
                         dev_status=status, **kw)
    torch.cuda.synchronize()
    return out.cpu()


def check(c, got, scale=None, max_q=None):
    dim, dtype = c["q"].shape[2], c["q"].dtype
    w = q4_plain.attention(c["q"], c["k"], c["v"], c["cu"], c["kv"], c["rows"], dim ** -0.5 if scale is None else scale)
    most = int(np.diff(c["cu"]).max()) if max_q is None else max_q
    many = most > 1 and most * (c["q"].shape[1] // c["k"][0].shape[1]) > 64
    with np.errstate(all="ignore"):
        bound = (q4_plain.bound_many if many else q4_plain.bound_rows)(w, dtype, dim, max(c["kv"] + [1]))
    got, out = got.double().numpy(), w["out"]
    assert np.array_equal(np.isfinite(got), np.isfinite(out))
    worst = np.max((np.abs(got - out) / bound)[np.isfinite(out)], initial=0.0)
    assert worst <= 1.0, f"error {worst:.2f} of its bound"


CASES = [
    # fresh, kv, hq, hkv, dim, dtype, page
    # single tokens
    ([1], [1], 1, 1, 64, BF, 16),
    ([1, 1, 1], [1, 16, 17], 8, 2, 128, BF, 16),
    ([1] * 5, [300, 1, 0, 64, 129], 32, 8, 128, BF, 64),
    ([1, 1], [1000, 2500], 16, 2, 128, FP, 32),
    ([1, 1], [700, 33], 40, 1, 64, FP, 128),       # more heads to a group than a tile's rows
    ([1, 1], [513, 255], 7, 1, 128, BF, 256),
    ([1] * 3, [128, 5, 777], 3, 3, 64, FP, 16),    # no groups
    ([1] * 2, [600, 601], 64, 4, 128, FP, 16),     # groups of sixteen
    ([1] * 2, [90, 61], 50, 2, 128, BF, 16),       # of twenty-five
    ([1] * 40, [40 + 7 * i for i in range(40)], 4, 2, 64, BF, 16),
    # drafted tokens
    ([2, 5, 3], [2, 77, 400], 8, 2, 128, BF, 16),
    ([5, 5], [900, 1200], 24, 8, 64, BF, 32),
    ([4], [641], 32, 4, 128, FP, 64),
    ([3, 1, 0, 2], [31, 32, 33, 34], 9, 3, 128, FP, 16),
    # chunks of prompts, mixed with single tokens
    ([17, 1, 128, 130], [17, 1, 128, 130], 4, 1, 128, BF, 16),
    ([255, 0, 257], [255, 0, 257], 2, 2, 64, BF, 32),
    ([128, 1, 40], [500, 333, 40], 8, 2, 128, BF, 16),
    ([64], [1087], 8, 8, 128, BF, 64),
    ([33, 200], [290, 201], 16, 2, 64, FP, 128),
    ([100], [613], 4, 1, 128, FP, 256),
    # fewer keys than tokens: the first rows see none
    ([5], [3], 4, 2, 128, BF, 16),
    ([200, 6], [130, 0], 4, 1, 128, BF, 32),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_64_bits(i):
    c = make(*CASES[i], seed=i)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check(c, call(c, status=status))
    assert int(status) == 0


@pytest.mark.parametrize("i", range(len(CASES)))
def test_wider_bounds_and_twice_the_same(i):
    c = make(*CASES[i], seed=i)
    wide = dict(max_kv=max(c["kv"]) + 1000)
    got = call(c, **wide)
    check(c, got)
    assert torch.equal(got, call(c, **wide))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fresh,kv,hq,hkv,dim,page", [
    ([1, 1], [9000, 5], 8, 1, 128, 16), ([1], [20000], 4, 4, 64, 64), ([1], [16385], 16, 1, 128, 128),
    ([3], [6001], 8, 1, 64, 16),
])
def test_long(dtype, fresh, kv, hq, hkv, dim, page):
    c = make(fresh, kv, hq, hkv, dim, dtype, page, seed=50)
    check(c, call(c))


@pytest.mark.parametrize("fresh,kv,hq,hkv,dim,dtype,page", [
    ([1] * 6, [9000, 5, 0, 1408, 1409, 5000], 8, 8, 128, BF, 16), ([2, 1, 2], [2, 9001, 3000], 32, 16, 128, FP, 64),
    ([1] * 4, [17000, 1, 1030, 4097], 16, 16, 64, BF, 128), ([3, 3], [17000, 900], 64, 16, 128, BF, 16),
])
def test_keys_in_chunks(fresh, kv, hq, hkv, dim, dtype, page):
    # long requests among short ones: their chunks are joined by a second kernel
    c = make(fresh, kv, hq, hkv, dim, dtype, page, seed=51)
    cache = cache_of(c)
    assert sss.sss_attention_q4_workspace_bytes(sum(fresh), hq, cache, len(kv), max(fresh), max(kv)) > 0
    got = call(c, cache=cache)
    check(c, got)
    assert torch.equal(got, call(c, cache=cache))


@pytest.mark.parametrize("n,most,hq,hkv,dim,dtype", [(64, 300, 8, 8, 64, FP), (44, 700, 128, 8, 128, BF), (320, 90, 1, 1, 128, BF)])
def test_more_requests_than_sms(n, most, hq, hkv, dim, dtype):
    # keys of a tile in one CTA
    c = make([1] * n, [(37 * i) % most for i in range(n)], hq, hkv, dim, dtype, 32, seed=52)
    check(c, call(c))


@pytest.mark.parametrize("fresh,kv,hq,hkv,dim", [
    ([700], [700], 56, 2, 64), ([13] * 41, [13 + i % 5 for i in range(41)], 32, 2, 128),
    ([70, 0, 1], [71, 500, 1], 48, 1, 128), ([3001], [3001], 5, 1, 64),
])
def test_more_rows_of_queries_than_of_keys(fresh, kv, hq, hkv, dim):
    c = make(fresh, kv, hq, hkv, dim, BF, 16, seed=53)
    check(c, call(c))


def test_pages_past_four_gigabytes():
    # a cache whose bytes are past 2^32, and a request whose pages lie at both of its ends;
    # one of them is copied to the far end first
    hq, hkv, dim, page = 8, 8, 128, 256
    pages = 2 ** 33 // (hkv * (page // 16) * 18 * dim) + 3
    cache = sss.empty_kv_cache_q4(pages, page, hkv, dim)
    c = make([1], [700], hq, hkv, dim, BF, page, seed=53, spare=0)
    near, far = [int(x) for x in c["table"][0, :3]], [pages - 1, 1, pages - 2]
    small = cache_of(c)
    for a, b in zip(near, far[:2] + [0]):
        cache.blocks[b] = small.blocks[a]
    one = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)  # noqa: E731
    sss.sss_page_copy(cache, one(0), one(far[2]))
    want = call(c)
    c["table"][0, :3] = torch.tensor(far, dtype=torch.int32)
    assert torch.equal(call(c, cache=cache), want)
    slots = torch.tensor(far[0] * page + np.arange(256), dtype=torch.int32, device=DEV)
    k, v = sss.sss_kv_fetch_q4(cache, slots)
    assert bool(torch.isfinite(k).all()) and float(k.abs().max()) > 0
    many = make([90], [700], hq, 1, dim, BF, page, seed=54, spare=0)  # (the copy for many rows, too)
    check(many, call(many))


def test_two_graphs_that_share_a_workspace():
    # replayed one after the other, each starts from whatever the other left there
    runs, ws = [], None
    for fresh, kv, hkv, dtype, seed in (([1] * 5, [9000, 30, 1500, 2048, 4097], 8, BF, 55), ([100, 60], [300, 700], 2, BF, 56),
                                        ([90], [500], 2, FP, 57)):
        c = make(fresh, kv, 8, hkv, 128, dtype, 16, seed=seed)
        runs.append((c, cache_of(c), call(c)))
    need = [sss.sss_attention_q4_workspace_bytes(sum(np.diff(c["cu"])), 8, cache, len(c["kv"]), int(np.diff(c["cu"]).max()),
                                                 max(c["kv"])) for c, cache, _ in runs]
    assert min(need) > 0
    ws = torch.empty(max(need), dtype=torch.uint8, device=DEV)
    graphs = []
    for c, cache, want in runs:
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        args = (c["q"].to(DEV), cache, ints(c["cu"]), ints(c["kv"]), int(np.diff(c["cu"]).max()), max(c["kv"]), c["table"].to(DEV))
        out, graph = torch.empty(c["q"].shape, dtype=c["q"].dtype, device=DEV), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sss.sss_attention_q4(*args, out=out, workspace=ws)
        graphs.append((graph, out, want, args))
    ws.fill_(0xFF)
    for i in (0, 1, 2, 1, 0, 2, 0, 0, 1):
        graph, out, want, _ = graphs[i]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("spread,scale", [(8.0, None), (1.0, 1e-6), (1.0, 3.0), (200.0, 1e-3), (1e-4, 50.0)])
def test_sharp_flat_and_far_scores(dtype, spread, scale):
    c = make([1, 2], [700, 90], 8, 2, 128, dtype, 16, seed=60, spread=spread)
    check(c, call(c, scale=scale), scale)


@pytest.mark.parametrize("dtype,spread", [(BF, 1e30), (BF, 1e-30), (FP, 60.0), (FP, 3e-6)])
def test_queries_at_the_ends_of_their_type(dtype, spread):
    # (the scores' scale undoes it)
    c = make([1, 1], [200, 33], 8, 2, 128, dtype, 16, seed=61, spread=spread)
    check(c, call(c, scale=0.1 / spread), 0.1 / spread)


def test_rows_of_unlike_size():
    # each row of q has its own range, a value in it far above the others
    c = make([1, 4], [300, 70], 6, 2, 128, BF, 16, seed=62)
    c["q"] *= (2.0 ** torch.arange(-15, 15)).repeat(1)[:c["q"].shape[0] * 6].view(-1, 6, 1).to(BF)
    c["q"][0, 1, 5], c["q"][2, 3, 100] = 1e5, -1e-4
    check(c, call(c, scale=1e-4), 1e-4)


def test_values_of_every_size():
    # scales from fp16's least to its largest
    c = make([1, 1], [64, 500], 8, 2, 64, BF, 16, seed=63)
    for name in "kv":
        u, s = c[name + "c"]
        g = np.random.default_rng(1)
        new = (np.exp2(g.integers(-24, -1 if name == "k" else 15, s.shape)) * g.choice([-1, 1], s.shape)).astype(np.float16)
        s[:] = new.view(np.uint16)
        c[name][0][c["slots"]], c[name][1][c["slots"]] = q4_plain.values(u, s), s
    check(c, call(c))


@pytest.mark.parametrize("fresh,kv,page", [([1, 1], [20, 700], 16), ([3], [40], 16), ([40], [100], 32)])
def test_tables_with_pages_that_are_none(fresh, kv, page):
    # such a page reads as zeros, flagged
    for bad in (-1, 10 ** 6, 2 ** 31 - 1):
        c = make(fresh, kv, 8, 2, 128, BF, page, seed=70)
        r = c["rows"](0)[:page]
        for name in "kv":
            c[name][0][r] = 0
            c[name][1][r] = 0
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        cache = cache_of(c)
        c["table"][0, 0] = bad
        got = call(c, status=status, cache=cache)
        c["rows"] = lambda b, first=c["rows"], r=r: np.concatenate([r, first(b)[page:]]) if b == 0 else first(b)
        check(c, got)
        assert int(status) == sss.FLAG_INDEX


def test_lengths_that_cannot_be():
    c = make([1, 1], [40, 50], 8, 2, 128, BF, 16, seed=71)
    cache, want = cache_of(c), call(c)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    # more keys than max_kv: cut to it, flagged, and the other request as it was
    c["kv"][1] = 5000
    got = call(c, status=status, max_kv=40, cache=cache)
    c["kv"][1] = 40
    check(c, got)
    assert int(status) == sss.FLAG_INDEX and torch.equal(got[0], want[0])
    c["kv"][1] = -3
    status.zero_()
    got = call(c, status=status, max_kv=50, cache=cache)
    assert int(status) == sss.FLAG_INDEX and not got[1].any()


@pytest.mark.parametrize("fresh", [[1, 3], [100, 20], [1]])
def test_no_keys_and_no_pages(fresh):
    # no keys at all: zeros; keys, but a cache without pages: zeros, flagged
    c = make(fresh, [0] * len(fresh), 8, 2, 64, BF, 16, seed=77)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for max_kv in (0, 500):
        assert not call(c, max_kv=max_kv, status=status).any() and int(status) == 0
    empty = sss.empty_kv_cache_q4(0, 16, 2, 64)
    c["kv"] = [max(fresh) + 5] * len(fresh)
    c["table"] = torch.zeros((len(fresh), 20), dtype=torch.int32)
    assert not call(c, cache=empty, status=status).any() and int(status) == sss.FLAG_INDEX


@pytest.mark.parametrize("cu", [[0, 3, 2, 6], [0, 2, 9, 9], [-1, 2, 4, 6], [0, 6, 6, 6]])
def test_tokens_that_cannot_be(cu):
    # requests that point past the tokens or backwards are left out, the others are right
    c = make([2, 2, 2], [20, 30, 40], 8, 2, 128, BF, 16, seed=78)
    cache, want = cache_of(c), call(c, max_q=6)
    c["cu"] = cu
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = call(c, cache=cache, max_q=6, status=status)
    for b in range(3):
        if cu[b] == 2 * b and cu[b + 1] == 2 * b + 2:
            assert torch.equal(got[2 * b:2 * b + 2], want[2 * b:2 * b + 2])
    assert int(status) == (0 if cu == [0, 6, 6, 6] else sss.FLAG_INDEX)


@pytest.mark.parametrize("many", [False, True])
def test_rows_of_no_request_are_left_alone(many):
    c = make([2, 3], [30, 70], 8 if many else 4, 1, 64, BF, 16, seed=72)
    want = call(c, max_q=5)
    c["q"] = torch.cat([c["q"], torch.full((4, c["q"].shape[1], 64), float("nan"), dtype=BF)])
    got = call(c, max_q=5)
    assert torch.equal(got[:5], want) and bool((got[5:] == 7).all())


def test_nan_and_infinite_queries_stay_in_their_rows():
    for value in (float("nan"), float("inf")):
        c = make([1, 1, 2], [40, 300, 20], 8, 2, 128, BF, 16, seed=73)
        want = call(c)
        c["q"][1, 3, 9] = value
        c["q"][3, 0, 2] = value
        got = call(c)
        for t in range(4):
            for h in range(8):
                if (t, h) in ((1, 3), (3, 0)):
                    assert bool(got[t, h].isnan().all())
                else:
                    assert torch.equal(got[t, h], want[t, h])


def test_keys_that_a_drafted_row_does_not_see():
    # whatever the later tokens' keys and values hold, scales of NaN and infinity among it
    c = make([4], [37], 4, 2, 128, BF, 16, seed=74)
    want = call(c)
    for scale in (0x7E00, 0x7C00, 0xFC00):
        for name in "kv":
            c[name + "c"][1][-1] = scale  # the last token's own
        got = call(c)
        assert torch.equal(got[:3], want[:3])


def test_strided_queries_another_stream_and_a_graph():
    for fresh, kv in (([1] * 6, [100, 900, 3, 17, 64, 2000]), ([40, 30], [400, 30])):
        c = make(fresh, kv, 8, 2, 128, BF, 16, seed=75)
        want, cache = call(c), cache_of(c)
        t = sum(fresh)
        wide = torch.full((t, 12, 128), float("nan"), dtype=BF, device=DEV)
        wide[:, 2:10] = c["q"].to(DEV)
        cu, kvl = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (c["cu"], c["kv"]))
        args = (cu, kvl, max(fresh), max(kv), c["table"].to(DEV))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = sss.sss_attention_q4(wide[:, 2:10], cache, *args, stream=side)
        side.synchronize()
        assert torch.equal(got.cpu(), want)
        q, out = c["q"].to(DEV), torch.zeros_like(got)
        need = sss.sss_attention_q4_workspace_bytes(t, 8, cache, len(kv), max(fresh), max(kv))
        ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sss.sss_attention_q4(q, cache, *args, out=out, workspace=ws)
        for _ in range(2):
            out.zero_()
            if ws is not None:
                ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), want)


def test_a_workspace_that_is_too_small():
    c = make([40], [100], 4, 2, 64, BF, 16, seed=76)
    with pytest.raises(sss.SssError, match="WORKSPACE"):
        call(c, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))


def test_python_refusals():
    c = make([1], [20], 4, 2, 64, BF, 16)
    cache = cache_of(c)
    q = c["q"].to(DEV)
    cu, kv, table = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 1], [20], [[0, 1]]))
    good = dict(q=q, cache=cache, cu_q=cu, kv_len=kv, max_q=1, max_kv=32, block_table=table)
    for change, what in ((dict(q=q.float()), "float16"), (dict(q=q[..., :32]), "dim"), (dict(q=q[0]), "must be"),
                         (dict(kv_len=None), "required"), (dict(block_table=None), "required"), (dict(kv_len=kv.long()), "int32"),
                         (dict(block_table=table[0]), "batch"), (dict(out=q.half()), "must be"), (dict(cu_q=cu[:0]), "batch"),
                         (dict(q=q.cpu()), "CUDA"), (dict(scale=0.0), "SSS_E_ARG"), (dict(max_kv=-1), "SSS_E_ARG"),
                         (dict(cache=sss.empty_kv_cache(2, 16, 2, 64)), "KVCacheQ4")):
        with pytest.raises(sss.SssError, match=what):
            sss.sss_attention_q4(**{**good, **change})
