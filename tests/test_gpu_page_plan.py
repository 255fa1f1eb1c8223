"""sss_page_plan against counting: whole numbers, equal to the last."""
import numpy as np
import pytest
import torch

import attn_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(v, shape=None):
    t = torch.tensor(v, dtype=torch.int32, device=DEV)
    return t if shape is None else t.reshape(shape)


def setup(past, fresh, page, spare=0, width=None, seed=0):
    rng = np.random.default_rng(seed)
    held = [-(-p // page) for p in past]
    total = [-(-(p + f) // page) for p, f in zip(past, fresh)]
    order = rng.permutation(sum(total) + spare)
    width = max(total + [0]) + 1 if width is None else width
    table = np.full((len(past), width), -7, np.int64)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:]


def call(past, fresh, page, free, table, tokens, stream=None):
    b = len(past)
    t = ints(table.tolist(), table.shape)
    cu, kv, used = ints([-9] * (b + 1)), ints([-9] * b), ints([-9])
    positions, slots, status = ints([-9] * tokens), ints([-9] * tokens), ints([0])
    sss.sss_page_plan(ints(past), ints(fresh), page, ints(list(free)), t, cu, kv, positions, slots, used,
                      dev_status=status, stream=stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, cu, kv, positions, slots, used)], int(status)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("past,fresh,spare,pad", [
    ([0], [1], 0, 0), ([5], [0], 3, 2), ([16, 15, 0, 31], [1, 1, 1, 1], 5, 0),
    ([0, 0, 100, 0, 64], [300, 0, 1, 257, 64], 1, 9), ([0] * 3, [0] * 3, 0, 4),
    (list(range(0, 1400, 2)), [i % 5 for i in range(700)], 11, 1),  # more than a chunk of requests
    ([7] * 257, [0] * 256 + [40], 0, 0),
    ([3, 250, 0], [20000, 1, 9000], 2, 0),                          # more tokens than a CTA's
])
def test_against_counting(page, past, fresh, spare, pad):
    table, free = setup(past, fresh, page, spare, seed=page)
    tokens = sum(fresh) + pad
    got, status = call(past, fresh, page, free, table, tokens)
    want = attn_plain.page_plan(past, fresh, page, free, table, tokens)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    assert status == 0


def test_no_requests():
    got, status = call([], [], 16, [3, 4], np.zeros((0, 4), np.int64), 3)
    assert status == 0 and got[1].tolist() == [0] and got[5].tolist() == [0]
    assert got[3].tolist() == [0] * 3 and got[4].tolist() == [-1] * 3


def test_called_again_it_says_the_same():
    past, fresh = [10, 0, 40], [30, 5, 1]
    table, free = setup(past, fresh, 16)
    first, _ = call(past, fresh, 16, free, table, 36)
    again, _ = call(past, fresh, 16, free, first[0], 36, stream=torch.cuda.Stream())
    for g, w in zip(again, first):
        assert np.array_equal(g, w)


def test_too_few_pages():
    past, fresh, page = [16, 0, 3], [16, 40, 1], 16
    table, free = setup(past, fresh, page)
    assert len(free) == 4  # one for request 0, three for request 1
    got, status = call(past, fresh, page, free[:3], table, 57)
    want = attn_plain.page_plan(past, fresh, page, free, table, 57)
    assert status == sss.FLAG_PAGES and got[5].tolist() == [3]
    want[0][1, 2] = -1            # request 1's last page
    want[4][16 + 32:16 + 40] = -1  # and its last eight tokens
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[4], want[4])
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])


def test_too_few_columns():
    past, fresh, page = [0, 0], [40, 16], 16
    table, free = setup(past, fresh, page)
    narrow = table[:, :2]
    got, status = call(past, fresh, page, free, narrow, 56)
    want = attn_plain.page_plan(past, fresh, page, free, table, 56)
    assert status == sss.FLAG_PAGES
    assert np.array_equal(got[0], want[0][:, :2])
    want[4][32:40] = -1
    assert np.array_equal(got[4], want[4])


def test_lengths_and_entries_that_cannot_be():
    # negative lengths count as none
    table, free = setup([0, 4], [3, 2], 16, spare=2)
    got, status = call([0, 4], [-5, 2], 16, free, table, 5)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [0, 0, 2]
    assert got[4].tolist()[2:] == [-1] * 3
    # a held page that is none
    table, free = setup([4], [2], 16)
    table[0, 0] = -1
    got, status = call([4], [2], 16, free, table, 2)
    assert status == sss.FLAG_INDEX and got[4].tolist() == [-1, -1]
    # more new tokens than the buffers have rows: cu_q ends there
    table, free = setup([0, 0], [3, 4], 16)
    got, status = call([0, 0], [3, 4], 16, free, table, 5)
    assert status == sss.FLAG_INDEX and got[1].tolist() == [0, 3, 5]
    want = attn_plain.page_plan([0, 0], [3, 4], 16, free, table, 7)
    assert np.array_equal(got[4], want[4][:5])
    # lengths whose sum is no int32
    _, status = call([2 ** 31 - 1], [5], 16, [0], np.full((1, 2), -1), 4)
    assert status & sss.FLAG_INDEX


def test_python_refusals():
    a = dict(past=ints([1]), fresh=ints([1]), page_size=16, free_pages=ints([1]), block_table=ints([[0, 0]]),
             cu_q=ints([0, 0]), kv_len=ints([0]), positions=ints([0]), slots=ints([0]), used=ints([0]))
    bad = [(dict(past=a["past"].long()), "int32"), (dict(fresh=ints([1, 2])), "elements"),
           (dict(cu_q=ints([0])), "elements"), (dict(slots=ints([0, 0])), "elements"),
           (dict(block_table=ints([0, 0])), "batch"), (dict(used=a["used"].cpu()), "CUDA"),
           (dict(page_size=24), "SSS_E_ARG"), (dict(page_size=0), "SSS_E_ARG")]
    for change, what in bad:
        with pytest.raises(sss.SssError, match=what):
            sss.sss_page_plan(**{**a, **change})
