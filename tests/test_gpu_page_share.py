"""sss_page_fork, sss_page_reclaim and sss_page_copy against going through the rows: whole
numbers and bytes, equal to the last."""
import numpy as np
import pytest
import torch

import q4_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(v, shape=None):
    t = torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device=DEV)
    return t if shape is None else t.reshape(shape)


def table_of(past, page, spare=0, seed=0, width=None, sparse=1.0):
    """A table whose rows hold their pages, in a random order, and pages that are free."""
    rng = np.random.default_rng(seed)
    held = [-(-p // page) for p in past]
    total = int((sum(held) + spare) * sparse)
    order = rng.permutation(total)
    width = max(held + [0]) + 1 if width is None else width
    table = np.full((len(past), width), -7, np.int64)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:], total


def call_fork(parents, past, page, free, table, stream=None):
    rows, width = len(parents), table.shape[1]
    new, lens, src, dst, used, status = (ints([-9] * n) for n in (rows * width, rows, rows, rows, 1, 1))
    status.zero_()
    new = new.reshape(rows, width)
    sss.sss_page_fork(ints(parents), ints(past), page, ints(free), ints(table, table.shape), new, lens, src, dst, used,
                      dev_status=status, stream=stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (new, lens, src, dst, used)], int(status)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("past,parents", [
    ([5], [0]), ([16], [0, 0, 0]), ([17], [0, 0, 0]), ([0], [0, 0]), ([1, 300, 0, 64], [3, 1, 1, 0, 0, 2, 1, -1, 1]),
    ([40, 41], []), ([7] * 40, list(range(39, -1, -1)) * 2),
    ([5000, 16, 33], [0, 1, 2, 0, 1, 2, 0]),
    ([1 + 3 * i for i in range(300)], [(7 * i) % 300 for i in range(700)]),  # more rows than a CTA looks at
    ([9], [0] * 600), ([33] * 2000, [i // 3 for i in range(1500)] + [1999] * 20),
])
def test_fork(page, past, parents):
    table, free, _ = table_of(past, page, spare=len(parents) + 3, seed=page)
    got, status = call_fork(parents, past, page, free, table)
    want = q4_plain.fork(parents, past, page, free, table)
    for g, w in zip(got, want):
        assert np.array_equal(g, w.reshape(g.shape))
    assert status == 0
    again, _ = call_fork(parents, past, page, free, table, stream=torch.cuda.Stream())
    for g, w in zip(again, got):
        assert np.array_equal(g, w)


def test_fork_with_too_few_pages():
    past, parents, page = [20, 40], [0, 0, 1, 0, 1, 1], 16
    table, free, _ = table_of(past, page, spare=4)
    want = q4_plain.fork(parents, past, page, free, table)
    for short in (free[:2], np.concatenate([free[:2], [-1, -1, -1]])):  # (-1: none, as reclaim leaves it)
        got, status = call_fork(parents, past, page, short, table)
        assert status == sss.FLAG_PAGES
        assert got[3].tolist() == [-1, free[0], -1, free[1], -1, -1]
        assert got[2].tolist() == [-1, table[0, 1], -1, table[0, 1], -1, -1]
        assert got[1].tolist() == [20, 20, 40, 20, 32, 32]
        assert got[0][4].tolist() == got[0][5].tolist() == [table[1, 0], table[1, 1], -1, -1]
        assert np.array_equal(got[0][:4], want[0][:4])


def test_fork_of_what_cannot_be():
    table, free, _ = table_of([20, 40], 16, spare=9)
    # a parent past the batch, a negative length, one that is longer than the row
    got, status = call_fork([0, 2, 1], [20, 40], 16, free, table)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [20, 0, 40] and got[0][1].tolist() == [-1] * 4
    got, status = call_fork([0, 1], [-3, 40], 16, free, table)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [0, 40]
    got, status = call_fork([0, 0], [100, 40], 16, free, table)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [64, 64] and got[2].tolist() == [-1, -1]
    # a last page to copy that is none: the row ends before it
    table[0, 1] = -1
    got, status = call_fork([0, 0], [20, 40], 16, free, table)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [20, 16] and got[3].tolist() == [-1, -1] and got[4].tolist() == [0]


def test_fork_of_nothing():
    got, status = call_fork([], [], 16, [3], np.zeros((0, 4), np.int64))
    assert status == 0 and got[4].tolist() == [0]
    got, status = call_fork([-1, -5], [], 16, [3], np.zeros((0, 4), np.int64))
    assert status == 0 and got[1].tolist() == [0, 0] and got[0].tolist() == [[-1] * 4] * 2


def call_reclaim(table, past, page, pages, most=None, in_place=False, stream=None):
    t, free, count, status = ints(table, table.shape), ints([-9] * pages), ints([-9]), ints([0])
    more, back = {}, []
    if most is not None:
        new = t if in_place else ints(np.full(table.shape, -7), table.shape)
        src, dst, moves = ints([-9] * most), ints([-9] * most), ints([-9])
        more, back = dict(new_table=new, src=src, dst=dst, moves=moves), [new, src, dst, moves]
    sss.sss_page_reclaim(t, ints(past), page, free, count, **more, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in [free, count] + back], int(status)


RECLAIM = [
    ([5], 16, 0, 1.0), ([0, 0], 16, 7, 1.0), ([17, 300, 0, 64], 16, 5, 2.0), ([4000, 16, 33], 16, 100, 3.0),
    ([33 * i for i in range(64)], 32, 1000, 1.5), ([2000] * 40, 16, 0, 1.0), ([1], 256, 99999, 1.0),
    ([9000 + 7 * i for i in range(150)], 16, 5000, 1.7),  # several CTAs
    ([16 * 1000] * 20, 16, 900000, 1.0),
]


@pytest.mark.parametrize("past,page,spare,sparse", RECLAIM)
def test_reclaim(past, page, spare, sparse):
    table, _, pages = table_of(past, page, spare, seed=3, sparse=sparse)
    got, status = call_reclaim(table, past, page, pages)
    want = q4_plain.reclaim(table, past, page, pages)
    assert status == 0
    for g, w in zip(got, want):
        assert np.array_equal(g, w)


@pytest.mark.parametrize("past,page,spare,sparse", RECLAIM)
@pytest.mark.parametrize("most", [0, 1, 50, 1 << 16])
@pytest.mark.parametrize("in_place", [False, True])
def test_reclaim_with_moves(past, page, spare, sparse, most, in_place):
    table, _, pages = table_of(past, page, spare, seed=4, sparse=sparse)
    table[len(past) // 2:, :1] = table[0, 0]  # a page that many hold
    got, status = call_reclaim(table, past, page, pages, most, in_place)
    want = q4_plain.reclaim(table, past, page, pages, most)
    if any(p == 0 for p in past):  # (entries behind a row's pages are left alone)
        keep = np.array(past) == 0
        got[2][keep] = want[2][keep]
    held = np.arange(table.shape[1])[None] < -(-np.array(past)[:, None] // page)
    for i, (g, w) in enumerate(zip(got, want)):
        if i == 2:
            assert np.array_equal(g[held], w[held])
            assert np.array_equal(g[~held], table[~held] if in_place else np.where(np.array(past)[:, None] == 0, w, -7)[~held])
        else:
            assert np.array_equal(g, w)
    # (where the first row holds nothing, what was put in the others' place is no page)
    assert status == (sss.FLAG_INDEX if (table[held] < 0).any() else 0)


def test_reclaim_of_nothing():
    got, status = call_reclaim(np.zeros((0, 3), np.int64), [], 16, 5, most=2)
    assert status == 0 and got[0].tolist() == [0, 1, 2, 3, 4] and got[1].tolist() == [5] and got[5].tolist() == [0]
    got, status = call_reclaim(np.zeros((0, 3), np.int64), [], 16, 0)
    assert status == 0 and got[1].tolist() == [0]
    # every page is held
    table = np.arange(6).reshape(2, 3)
    got, status = call_reclaim(table, [48, 48], 16, 6, most=4)
    assert status == 0 and got[0].tolist() == [-1] * 6 and got[1].tolist() == [0] and got[5].tolist() == [0]


def test_reclaim_of_what_cannot_be():
    table = np.array([[3, -1, 9], [40, 2, 5]])
    got, status = call_reclaim(table, [48, 33], 16, 10, most=3)
    assert status == sss.FLAG_INDEX
    # pages 2, 3, 5 and 9 are held: 9 -> 0, 5 -> 1
    assert got[3].tolist() == [9, 5, -1] and got[4].tolist() == [0, 1, -1] and got[1].tolist() == [6]
    assert got[2].tolist() == [[3, -1, 0], [40, 2, 1]] and got[0].tolist() == [4, 5, 6, 7, 8, 9, -1, -1, -1, -1]
    got, status = call_reclaim(np.array([[3, 1]]), [-5], 16, 4)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [4]
    got, status = call_reclaim(np.array([[3, 1]]), [1000], 16, 4)
    assert status == sss.FLAG_INDEX and got[0].tolist() == [0, 2, -1, -1]


def caches_of(form, layers, pages, page, heads, dim, seed=0, strided=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    for _ in range(layers):
        if form == "q4":
            shape = (pages, 2 * heads if strided else heads, page // 16, 18 * dim)
            t = torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8)
            out.append(sss.KVCacheQ4(t[:, heads:] if strided else t))
        else:
            m = torch.randn((pages * page, (3 if strided else 2) * heads, dim), generator=g, device=DEV).to(form)
            out.append(sss.KVCache(m[:, :heads], m[:, -heads:], page) if strided else
                       sss.KVCache(m[:, :heads].contiguous(), m[:, heads:].contiguous(), page))
    return out


def parts(c):
    return [c.blocks] if isinstance(c, sss.KVCacheQ4) else [c.k, c.v]


@pytest.mark.parametrize("form", ["q4", torch.bfloat16, torch.float16])
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("layers,pages,page,heads,dim,n", [
    (1, 2, 16, 1, 64, 1), (3, 40, 16, 8, 128, 17), (2, 30, 256, 5, 64, 9), (128, 6, 16, 1, 128, 3), (1, 300, 64, 8, 128, 140),
])
def test_copy(form, strided, layers, pages, page, heads, dim, n):
    caches = caches_of(form, layers, pages, page, heads, dim, strided=strided)
    order = np.random.default_rng(n).permutation(pages)
    src, dst = order[:n].copy(), order[n:2 * n].copy()
    if n > 4:
        src[::5] = dst[::5] = -1
    want = []
    for c in caches:
        for x in parts(c):
            y = x.clone()
            z = y.unflatten(0, (pages, -1))
            for a, b in zip(src, dst):
                if a >= 0:
                    z[b] = z[a]
            want.append(y)
    status = ints([0])
    sss.sss_page_copy(caches, ints(src), ints(dst), dev_status=status)
    assert int(status) == 0
    for x, y in zip([x for c in caches for x in parts(c)], want):
        assert torch.equal(x, y)


def test_copy_leaves_the_rest_of_strided_pages():
    m = torch.randn((4 * 16, 6, 64), device=DEV).bfloat16()
    before = m.clone()
    sss.sss_page_copy(sss.KVCache(m[:, :2], m[:, 4:], 16), ints([3]), ints([1]))
    assert torch.equal(m[:, 2:4], before[:, 2:4]) and torch.equal(m[16:32, :2], before[48:, :2])


@pytest.mark.parametrize("form", ["q4", torch.bfloat16])
def test_copy_of_what_cannot_be(form):
    (c,) = caches_of(form, 1, 5, 16, 2, 64)
    before = [x.clone() for x in parts(c)]
    for a, b in ((0, 5), (5, 0), (-1, 2), (2, -1), (2 ** 31 - 1, 1), (-2 ** 31, 3)):
        status = ints([0])
        sss.sss_page_copy(c, ints([a]), ints([b]), dev_status=status)
        assert int(status) == sss.FLAG_INDEX
    status = ints([0])
    sss.sss_page_copy([c], ints([-1, -5]), ints([-3, -1]), dev_status=status)
    sss.sss_page_copy([], ints([0]), ints([1]), dev_status=status)
    sss.sss_page_copy([c], ints([]), ints([]), dev_status=status)
    assert int(status) == 0
    for x, y in zip(parts(c), before):
        assert torch.equal(x, y)


def test_python_refusals():
    table, past = ints(np.zeros((2, 3)), (2, 3)), ints([5, 6])
    a = dict(parents=ints([0, 1, 1]), past=past, page_size=16, free_pages=ints([9]), block_table=table,
             new_table=ints(np.zeros((3, 3)), (3, 3)), new_past=ints([0] * 3), src=ints([0] * 3), dst=ints([0] * 3), used=ints([0]))
    for change, what in ((dict(new_table=table), "must be"), (dict(src=ints([0])), "elements"), (dict(past=past.long()), "int32"),
                         (dict(block_table=ints([0] * 6)), "must be"), (dict(used=ints([0]).cpu()), "CUDA"),
                         (dict(page_size=24), "SSS_E_ARG")):
        with pytest.raises(sss.SssError, match=what):
            sss.sss_page_fork(**{**a, **change})
    same = {**a, "parents": ints([0, 1]), "new_table": table, "new_past": ints([0] * 2), "src": ints([0] * 2), "dst": ints([0] * 2)}
    with pytest.raises(sss.SssError, match="SSS_E_ARG"):  # rows would be read after they are written
        sss.sss_page_fork(**same)
    r = dict(block_table=table, past=past, page_size=16, free_pages=ints([0] * 9), free_count=ints([0]), new_table=table,
             src=ints([0]), dst=ints([0]), moves=ints([0]))
    for change, what in ((dict(new_table=None), "new_table"), (dict(dst=ints([0, 0])), "size"), (dict(moves=None), "required"),
                         (dict(new_table=table[:, :2]), "must be"), (dict(free_count=ints([])), "elements")):
        with pytest.raises(sss.SssError, match=what):
            sss.sss_page_reclaim(**{**r, **change})
    c16, q4 = sss.empty_kv_cache(2, 16, 1, 64), sss.empty_kv_cache_q4(2, 16, 1, 64)
    for caches, what in (([c16, q4], "KVCache"), ([q4, c16], "KVCacheQ4"), ([3], "KVCache"),
                         ([c16, sss.empty_kv_cache(3, 16, 1, 64)], "SSS_E_ARG"), ([c16] * 129, "SSS_E_ARG")):
        with pytest.raises(sss.SssError, match=what):
            sss.sss_page_copy(caches, ints([0]), ints([1]))
    with pytest.raises(sss.SssError, match="elements"):
        sss.sss_page_copy(c16, ints([0]), ints([1, 0]))
