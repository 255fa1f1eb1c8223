"""sss_page_fork of rows whose lengths were cut into pages that they share with others: no two
rows of the new table write to one page, whoever their parents are."""
import numpy as np
import pytest
import torch

import fork_plain
from paper_2607_08779_gb300 import sss
from test_gpu_page_share import call_fork, ints

pytestmark = pytest.mark.gpu
DEV = "cuda"


def shared_table(rng, batch, page, width, share):
    """Rows in families whose first pages are the same, and pages that are free."""
    table = rng.permutation(batch * width).reshape(batch, width)
    for b in range(batch):
        table[b, :share[b]] = table[b - b % 4, :share[b]]
    free = np.arange(batch * width, 2 * batch * width)
    return table, rng.permutation(free)


def check(parents, past, page, free, table):
    got, status = call_fork(parents, past, page, free, table)
    want = fork_plain.fork(parents, past, page, free, table)
    for g, w in zip(got, want):
        assert np.array_equal(g, w.reshape(g.shape))
    assert status == 0


@pytest.mark.parametrize("past,parents", [
    ([10, 10], [0, 1]), ([10, 20], [0, 1]), ([20, 10], [0, 1]), ([10, 20], [1, 0]), ([16, 10], [0, 1, 1, 0]),
    ([10, 10], [1, 1]), ([10, 5], [1, 0, 1, 0]), ([10, 31], [0, -1]), ([0, 3], [1, 0, 1]),
])
def test_two_rows_that_share_a_page(past, parents):
    check(parents, past, 16, [9, 8, 2, 1], np.array([[5, 6], [5, 7]]))


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("batch,rows,width,page", [(4, 4, 3, 16), (8, 40, 9, 32), (64, 200, 40, 16), (300, 1500, 17, 16),
                                                   (64, 512, 700, 16), (9, 30, 5000, 16), (256, 256, 300, 64)])
def test_families_cut_anywhere(seed, batch, rows, width, page):
    rng = np.random.default_rng(seed)
    share = rng.integers(0, width + 1, batch)
    table, free = shared_table(rng, batch, page, width, share)
    # cut around the point where a row leaves its family
    past = np.clip(share * page + rng.integers(-2 * page, 2 * page, batch), 0, width * page).astype(int)
    if seed % 2:
        past[:] = past[0]
    parents = np.arange(batch)[:rows] if seed % 3 == 0 else rng.integers(-1, batch, rows)
    check(parents.tolist(), past.tolist(), page, free, table)


@pytest.mark.parametrize("rows", [8192, 8193, 20000, 65535])
def test_more_rows_than_a_table_of_their_pages_holds(rows):
    # every row cut into a page that it shares with the next one or one far away
    rng = np.random.default_rng(rows)
    table = np.stack([rng.permutation(rows) // 2, rows + rng.permutation(rows) // 3], 1)
    past = rng.integers(0, 33, rows)
    check(rng.permutation(rows).tolist(), past.tolist(), 16, np.arange(2 * rows, 4 * rows), table)


def test_pages_that_are_none_among_those_that_are_shared():
    # -1 is no page: it is kept by each parent's first row, and not to be copied
    table = np.array([[-1, 3], [-1, 4], [3, -1]])
    got, status = call_fork([0, 1, 1, 2], [7, 9, 30], 16, [20, 21], table)
    assert status == sss.FLAG_INDEX
    assert got[1].tolist() == [7, 9, 0, 30] and got[2].tolist() == [-1] * 4 and got[4].tolist() == [0]
    assert got[0].tolist() == [[-1, -1], [-1, -1], [-1, -1], [3, -1]]


def test_rows_that_were_rolled_back_write_apart():
    # two requests forked from one, both cut into a page that they share, then one new token each:
    # what each reads back is its own
    heads, dim, page = 2, 64, 16
    g = torch.Generator(device=DEV).manual_seed(5)
    normal = lambda n: torch.randn((n, heads, dim), generator=g, device=DEV)  # noqa: E731
    cache, status = sss.empty_kv_cache_q4(12, page, heads, dim), ints([0])
    cache.blocks.zero_()
    table = ints([[3, 4, 5], [3, 4, 6]])
    start = normal(48)
    slots = torch.cat([table[0].repeat_interleave(page) * page + torch.arange(48, device=DEV) % page]).int()
    sss.sss_kv_store_q4(start, start, cache, slots)
    for past in ([20, 20], [20, 47], [47, 20]):
        new, lens, src, dst, used = ints([[-1] * 3] * 2), ints([0, 0]), ints([0, 0]), ints([0, 0]), ints([0])
        before = [sss.sss_kv_fetch_q4(cache, (table[b].repeat_interleave(page) * page + torch.arange(48, device=DEV) % page)
                                      .int()[:n])[0] for b, n in enumerate(past)]
        sss.sss_page_fork(ints([0, 1]), ints(past), page, ints([7, 8, 9]), table, new, lens, src, dst, used, dev_status=status)
        sss.sss_page_copy(cache, src, dst, dev_status=status)
        cu, kv, positions, to = ints([0] * 3), ints([0] * 2), ints([0, 0]), ints([0, 0])
        sss.sss_page_plan(lens, ints([1, 1]), page, ints([10, 11]), new, cu, kv, positions, to, used, dev_status=status)
        x = normal(2)
        sss.sss_kv_store_q4(x, x, cache, to, dev_status=status)
        held = sss.sss_kv_fetch_q4(cache, to)[0]
        assert len(set(to.tolist())) == 2 and not torch.equal(held[0], held[1])
        for b, n in enumerate(past):
            where = (new[b].repeat_interleave(page) * page + torch.arange(48, device=DEV) % page).int()[:n + 1]
            got = sss.sss_kv_fetch_q4(cache, where)[0]
            assert torch.equal(got[:n], before[b]) and torch.equal(got[n], held[b])
        assert int(status) == 0
        sss.sss_kv_store_q4(start, start, cache, slots)


def test_tables_without_columns_and_wide_ones():
    got, status = call_fork([0, 0, 1], [0, 0], 16, [3], np.zeros((2, 0), np.int64))
    assert status == 0 and got[1].tolist() == [0, 0, 0] and got[4].tolist() == [0]
    got, status = call_fork([0], [5], 16, [3], np.zeros((1, 0), np.int64))
    assert status == sss.FLAG_INDEX and got[1].tolist() == [0]
    rng = np.random.default_rng(7)
    table = rng.permutation(600000).reshape(2, 300000)
    table[1, :200000] = table[0, :200000]
    for past in ([16 * 200000 - 3, 16 * 199999 + 2], [16 * 250000 + 1, 16 * 100000 + 7], [16 * 300000, 16 * 300000 - 1]):
        check([0, 1, 0], past, 16, np.arange(600000, 600010), table)
