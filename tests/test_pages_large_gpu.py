"""Pages of a pool at the largest numbers that the calls take: many sequences, as many pages and moves as an int counts."""
import numpy as np
import pytest
import torch

from paper_2407_08608_amd import binding
from test_pages_gpu import _ints, _same

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def _memory_goes_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("last", [16, 5])
def test_fork_of_millions(last):
    """The work goes by the new sequences' entries, not by their number times the old ones'"""
    B, n_pages = 1 << 21, 3 << 20
    g = np.random.default_rng(last)
    page = g.permutation(n_pages)[:B]
    parents = g.permutation(B)
    parents[B // 2:B // 2 + 1000] = parents[:1000]  # these need a copy where the page is not full
    got = binding.fa_cache_fork(_ints(page[:, None]), _ints(np.full(B, last)), _ints(parents), 16, n_pages)
    rows, src, dst = page[parents], np.full(B, -1), np.full(B, -1)
    if last < 16:
        free = np.setdiff1d(np.arange(n_pages), rows)[:1000]
        src[B // 2:B // 2 + 1000], dst[B // 2:B // 2 + 1000] = rows[:1000], free
        rows = np.where(dst >= 0, dst, rows)
    _same(got, (rows, np.full(B, last), src, dst, 0))


def test_as_many_moves_as_an_int_counts():
    table = [[7, -1, 5], [2, 0, 9]]
    new, src, dst, top = binding.fa_cache_compact(_ints(table), 10, moves=MOST)
    assert new.tolist() == [[3, -1, 4], [2, 0, 1]] and src[:4].tolist() == [9, 7, 5, -1] and dst[:4].tolist() == [1, 3, 4, -1] and top.item() == 5
    for x in (src, dst):
        assert len(x) == MOST and all((part == -1).all() for part in x[3:].split(1 << 28))


@pytest.mark.parametrize("n_pages", [MOST, MOST - 2 ** 18 + 2, MOST - 2 ** 18 + 1])
def test_as_many_pages_as_an_int_counts(n_pages):
    # the last window of pages begins, ends, or would have a next one begin, past the last number but one
    last = n_pages - 1
    space = torch.empty(binding.fa_cache_pages_workspace_bytes(3, n_pages), dtype=torch.uint8, device="cuda")
    table = [[last, last - 1, -1], [0, last, 1], [2 ** 30, -1, -1]]
    got = binding.fa_cache_fork(_ints(table), _ints([20, 48, 9]), _ints([0, 0, 2]), 16, n_pages, workspace=space)
    _same(got, ([[last, last - 1, -1], [last, 0, -1], [2 ** 30, -1, -1]], [20, 20, 9], [-1, last - 1, -1], [-1, 0, -1], 0))
    got = binding.fa_cache_extend(_ints(table), _ints([20, 48, 9]), 24, 16, n_pages, workspace=space)
    _same(got, ([[last, last - 1, 2], [0, last, 1], [2 ** 30, 3, 4]], 2))
    got = binding.fa_cache_compact(_ints(table), n_pages, moves=5, workspace=space)
    _same(got, ([[2, 3, -1], [0, 2, 1], [4, -1, -1]], [last, last - 1, 2 ** 30, -1, -1], [2, 3, 4, -1, -1], 5))
