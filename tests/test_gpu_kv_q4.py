"""sss_kv_store_q4 and sss_kv_fetch_q4 against the oracle's quantizer and the layout's
definition: bytes and values, equal to the last."""
import numpy as np
import pytest
import torch

import q4_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def filled(pages, page, heads, dim, fill=0xA5):
    c = sss.empty_kv_cache_q4(pages, page, heads, dim)
    c.blocks.fill_(fill)
    return c


def heads_of(n, heads, dim, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, dim), generator=g) * torch.exp(torch.randn((1, heads, dim), generator=g)) * scale
    return x.to(dtype)


def expect(k, v, slots, c):
    pages, heads, blocks, size = c.blocks.shape
    packed = [q4_plain.quantize(x.float().numpy()) for x in (k, v)]
    return q4_plain.blocks(packed[0][:2], packed[1][:2], slots, pages, 16 * blocks, heads, size // 18)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens,heads,page", [(1, 1, 16), (5, 3, 16), (37, 8, 32), (64, 5, 64), (130, 2, 256)])
def test_bytes_and_values(dtype, dim, tokens, heads, page):
    pages = -(-tokens // page) + 2
    k, v = (heads_of(tokens, heads, dim, dtype, seed=i) for i in (1, 2))
    slots = np.random.default_rng(tokens).permutation(pages * page)[:tokens].tolist()
    c = filled(pages, page, heads, dim)
    status = ints([0])
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), c, ints(slots), dev_status=status)
    assert np.array_equal(c.blocks.cpu().numpy(), expect(k, v, slots, c)) and int(status) == 0
    for out in DTYPES:
        got = sss.sss_kv_fetch_q4(c, ints(slots), dtype=out, dev_status=status)
        for x, g in zip((k, v), got):
            want = torch.from_numpy(q4_plain.on_grid(x.float().numpy())).float()  # exact in fp32
            assert g.dtype is out and torch.equal(g.cpu().float(), want.to(out).float())
    assert int(status) == 0


def test_slots_that_are_not_kept_or_not_there():
    k, v = (heads_of(6, 2, 64, torch.bfloat16, seed=i) for i in (3, 4))
    c, status = filled(3, 16, 2, 64), ints([0])
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), c, ints([5, -1, 47, -7, 0, 16]), dev_status=status)
    want = expect(k, v, [5, -1, 47, -7, 0, 16], c)
    assert np.array_equal(c.blocks.cpu().numpy(), want) and int(status) == 0
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), c, ints([5, -1, 47, 48, 0, 2 ** 31 - 1]), dev_status=status)
    assert int(status) == sss.FLAG_INDEX
    # the same slot may be fetched twice; a negative one gives zeros, as one past the cache does
    status.zero_()
    got, _ = sss.sss_kv_fetch_q4(c, ints([47, -1, 47, 5]), dev_status=status)
    kk = torch.from_numpy(q4_plain.on_grid(k.float().numpy())).float()
    assert torch.equal(got.cpu(), torch.stack([kk[2], 0 * kk[0], kk[2], kk[0]])) and int(status) == 0
    got, _ = sss.sss_kv_fetch_q4(c, ints([48, 47]), dev_status=status)
    assert torch.equal(got.cpu()[0], 0 * kk[0]) and torch.equal(got.cpu()[1], kk[2]) and int(status) == sss.FLAG_INDEX


def test_no_slots_given_no_tokens_and_one_side():
    k, v = (heads_of(20, 3, 128, torch.float16, seed=i) for i in (5, 6))
    c = filled(2, 16, 3, 128)
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), c)
    assert np.array_equal(c.blocks.cpu().numpy(), expect(k, v, list(range(20)), c))
    sss.sss_kv_store_q4(k[:0].to(DEV), v[:0].to(DEV), c, ints([]))
    less, status = filled(1, 16, 3, 128), ints([0])  # more tokens than slots
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), less, dev_status=status)
    assert int(status) == sss.FLAG_INDEX
    assert np.array_equal(less.blocks.cpu().numpy(), expect(k[:16], v[:16], list(range(16)), less))
    only = torch.full((2, 3, 128), 9.0, device=DEV)
    a, b = sss.sss_kv_fetch_q4(c, ints([3, 19]), v=only)
    assert a is None and b is only
    assert torch.equal(only.cpu(), torch.from_numpy(q4_plain.on_grid(v.float().numpy()))[[3, 19]].float())
    a, b = sss.sss_kv_fetch_q4(c, ints([]))
    assert a.shape == b.shape == (0, 3, 128)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_rows_and_pages(dtype):
    # k and v as columns of one matrix; the caches of two layers in one buffer
    m = heads_of(9, 1, 1024, dtype, seed=7).view(9, 1024).to(DEV)
    k, v = m[:, 256:512], m[:, 640:896]
    buffer = torch.full((4, 2, 2, 1, 18 * 128), 0x5A, dtype=torch.uint8, device=DEV)
    c = sss.KVCacheQ4(buffer[:, 1])
    slots = [60, 1, 33, 2, 3, 16, 15, 31, 47]
    sss.sss_kv_store_q4(k, v, c, ints(slots))
    packed = [q4_plain.quantize(x.float().cpu().numpy().reshape(9, 2, 128))[:2] for x in (k, v)]
    want = q4_plain.blocks(*packed, slots, 4, 16, 2, 128, fill=0x5A)
    assert np.array_equal(buffer[:, 1].cpu().numpy(), want) and bool((buffer[:, 0] == 0x5A).all())
    got, _ = sss.sss_kv_fetch_q4(c, ints(slots))
    assert np.array_equal(got.cpu().numpy(), q4_plain.values(*packed[0]).astype(np.float32))


def test_groups_that_are_hard():
    # ties of sign and of rounding, zeros of both signs, one value, tiny and huge ones
    rows = np.zeros((12, 1, 64), np.float32)
    rows[0, 0, :4] = [3.0, -3.0, 1.5, -0.1875]          # a tie keeps s > 0; halves of a step
    rows[1, 0, :] = -0.0
    rows[2, 0, 7] = 1e-7                                 # s below fp16's least: codes, scale 0
    rows[3, 0, 33] = -5e-42                              # subnormal
    rows[4, 0, :] = np.linspace(-8, 8, 64) * 65504       # just in range
    rows[5, 0, 3] = 600000.0                             # a scale of 75000
    rows[6, 0, 40] = -3e38
    rows[7, 0, :32] = np.arange(32) * 0.5 - 8            # every half step
    rows[8, 0, 5] = np.inf
    rows[9, 0, 5], rows[9, 0, 50] = np.nan, 2.0
    rows[10, 0, :] = 2.0 ** -24 * np.arange(64)
    rows[11, 0, 2], rows[11, 0, 3] = -np.inf, np.nan
    for part, flag in ((rows[:5], 0), (rows[5:7], sss.FLAG_RANGE), (rows[7:8], 0), (rows[8:10], sss.FLAG_NONFINITE),
                       (rows[10:11], 0), (rows[11:], sss.FLAG_NONFINITE)):
        x = torch.from_numpy(part)
        c, status = filled(1, 16, 1, 64), ints([0])
        sss.sss_kv_store_q4(x.to(DEV), x.to(DEV), c, dev_status=status)
        assert np.array_equal(c.blocks.cpu().numpy(), expect(x, x, list(range(len(part))), c))
        assert int(status) == flag
        got, _ = sss.sss_kv_fetch_q4(c, ints(list(range(len(part)))))
        assert bool(torch.isfinite(got).all())


def test_slots_past_two_gigabytes():
    # a cache whose bytes are past 2^32, and pages far apart
    heads, dim, page = 8, 128, 256
    per = heads * (page // 16) * 18 * dim
    pages = 2 ** 33 // per + 2
    c = sss.empty_kv_cache_q4(pages, page, heads, dim)
    k, v = (heads_of(2, heads, dim, torch.bfloat16, seed=i) for i in (8, 9))
    slots = [pages * page - 1, 5]
    sss.sss_kv_store_q4(k.to(DEV), v.to(DEV), c, ints(slots))
    a, b = sss.sss_kv_fetch_q4(c, ints(slots))
    for x, g in ((k, a), (v, b)):
        assert torch.equal(g.cpu().double(), torch.from_numpy(q4_plain.on_grid(x.float().numpy())))


def test_on_another_stream_and_captured():
    k, v = (heads_of(40, 4, 128, torch.bfloat16, seed=i).to(DEV) for i in (10, 11))
    c, slots = filled(4, 16, 4, 128), ints(list(range(63, 23, -1)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sss.sss_kv_store_q4(k, v, c, slots, stream=side)
    a, b = sss.sss_kv_fetch_q4(c, slots, dtype=torch.bfloat16, stream=side)
    side.synchronize()
    once = c.blocks.clone()
    graph = torch.cuda.CUDAGraph()
    a2, b2 = torch.empty_like(a), torch.empty_like(b)
    with torch.cuda.graph(graph):
        sss.sss_kv_store_q4(k, v, c, slots)
        sss.sss_kv_fetch_q4(c, slots, a2, b2)
    c.blocks.fill_(0xA5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.blocks, once) and torch.equal(a, a2) and torch.equal(b, b2)


def test_python_refusals():
    c = filled(2, 16, 2, 64)
    k = torch.zeros((3, 2, 64), device=DEV)
    s = ints([0, 1, 2])
    for f, what in ((lambda: sss.sss_kv_store_q4(k, k.half(), c, s), "dtype"),
                    (lambda: sss.sss_kv_store_q4(k.double(), k.double(), c, s), "dtype"),
                    (lambda: sss.sss_kv_store_q4(k[:2], k, c, s), "must be"),
                    (lambda: sss.sss_kv_store_q4(k, k, c, s[:2]), "elements"),
                    (lambda: sss.sss_kv_store_q4(k, k, c, s.long()), "int32"),
                    (lambda: sss.sss_kv_store_q4(k.cpu(), k.cpu(), c, s), "CUDA"),
                    (lambda: sss.sss_kv_store_q4(k[..., ::2], k, c, s), "must be"),
                    (lambda: sss.sss_kv_store_q4(k, k, sss.empty_kv_cache(2, 16, 2, 64), s), "KVCacheQ4"),
                    (lambda: sss.sss_kv_fetch_q4(c, s, k, k.half()), "must be"),
                    (lambda: sss.sss_kv_fetch_q4(c, s, k, dtype=torch.float16), "dtype"),
                    (lambda: sss.sss_kv_fetch_q4(c, s, k[:2]), "elements"),
                    (lambda: sss.sss_kv_fetch_q4(c, s.long()), "int32"),
                    (lambda: sss.sss_kv_fetch_q4(c, s.cpu()), "CUDA")):
        with pytest.raises(sss.SssError, match=what):
            f()
