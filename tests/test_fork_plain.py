"""The plain fork that sss_page_fork is compared with, on tables worked out by hand."""
import numpy as np
import pytest

import fork_plain
import q4_plain


def lists(*args):
    return [x.tolist() for x in fork_plain.fork(*args)]


def test_rows_cut_into_a_page_that_they_share():
    # two beams share page 5, which was full: both are cut to its middle
    table = np.array([[5, 6], [5, 7]])
    assert lists([0, 1], [10, 10], 16, [9, 8], table) == [[[5, -1], [9, -1]], [10, 10], [-1, 5], [-1, 9], [1]]
    # one alone is cut: the other still holds all of it
    assert lists([0, 1], [10, 20], 16, [9, 8], table) == [[[9, -1], [5, 7]], [10, 20], [5, -1], [9, -1], [1]]
    assert lists([1, 0], [10, 20], 16, [9, 8], table) == [[[5, 7], [9, -1]], [20, 10], [-1, 5], [-1, 9], [1]]
    # both full: shared; a row that nobody takes over has no say
    assert lists([0, 1], [16, 16], 16, [9], table) == [[[5, -1], [5, -1]], [16, 16], [-1, -1], [-1, -1], [0]]
    assert lists([0, 0], [10, 20], 16, [9], table) == [[[5, -1], [9, -1]], [10, 10], [-1, 5], [-1, 9], [1]]


@pytest.mark.parametrize("seed", range(20))
def test_without_a_cut_it_is_by_parents(seed):
    rng = np.random.default_rng(seed)
    past = rng.integers(0, 100, 7)
    table = rng.permutation(70).reshape(7, 10)
    parents = rng.integers(-1, 7, 20).tolist()
    free = np.arange(100, 130)
    for a, b in zip(fork_plain.fork(parents, past, 16, free, table), q4_plain.fork(parents, past, 16, free, table)):
        assert np.array_equal(a, b)
