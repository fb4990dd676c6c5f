"""Pages of a pool where their holders, their numbers or their tables are not the usual ones: what the oracle gives, and what a cache then holds."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle
from paper_2407_08608_amd import binding
from test_pages_gpu import _ints, _same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [40, 5000])
@pytest.mark.parametrize("copies", [1, 3, 1100])
def test_a_held_page_that_is_not_full_is_copied(n_pages, copies):
    n = max(n_pages, copies + 10)
    table, lens = [[0, 1, -1], [7, 5, 6]], [20, 33]
    for pages in ([], [0, 1], [1], [6], [0, 1, 5, 6, 7]):
        held = np.zeros(n, dtype=np.int64)
        held[pages] = 3
        for parents in ([0] * copies, [1, 0] * copies):
            _same(binding.fa_cache_fork(_ints(table), _ints(lens), _ints(parents), 16, n, held=_ints(held)), pages_oracle.fork(table, lens, parents, held, 16, n))


def test_two_batches_that_go_on_from_one_prompt():
    """Two tables of one pool, each forked from the same stored prompt in a call of its own, each with all that the other and the store have held:
    what each writes and reads back is its own, and the prompt stays"""
    H_kv, page, d, n_pages, wide, prompt = 2, 16, 64, 24, 4, 20
    k, v = (torch.zeros((n_pages, H_kv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    said = torch.randn((2, 1, H_kv, prompt, d), device="cuda").bfloat16()
    store = _ints([[4, 9] + [-1] * (wide - 2)])
    binding.fa_cache_write(said[0], said[1], k, v, store, _ints([0]))
    held = np.zeros(n_pages, dtype=np.int64)
    held[[4, 9]] = 1
    batches = []
    for beams in (1, 3):
        table, lens, src, dst, missing = binding.fa_cache_fork(store, _ints([prompt]), _ints([0] * beams), page, n_pages, held=_ints(held))
        binding.fa_cache_copy(k, v, src, dst)
        table, none = binding.fa_cache_extend(table, lens, 9, page, n_pages, held=_ints(held))
        assert missing.item() == 0 and none.item() == 0
        held[[p for p in table.flatten().tolist() if p >= 0]] = 1
        batches.append((table, lens, torch.randn((2, beams, H_kv, 9, d), device="cuda").bfloat16()))
    for table, lens, new in batches:
        binding.fa_cache_write(new[0], new[1], k, v, table, lens)
    for table, lens, new in batches:
        got = binding.fa_cache_read(k, v, table, lens + 9, N=prompt + 9)
        for x, old, more in zip(got, said, new):
            assert torch.equal(x[:, :, :prompt], old.expand(table.shape[0], -1, -1, -1)) and torch.equal(x[:, :, prompt:], more)
    for x, old in zip(binding.fa_cache_read(k, v, store, _ints([prompt]), N=prompt), said):
        assert torch.equal(x, old)


@pytest.mark.parametrize("n", [2 ** 23 - 1, 2 ** 23, 2 ** 23 + 5, 3 * 2 ** 23])
def test_more_pairs_than_a_launch_takes(n):
    # small pages, a pair to two workgroups: a grid ends at 2^23 - 1 pairs
    n_pages = 40
    g = torch.Generator(device="cuda").manual_seed(n % 1000)
    have = [torch.randint(0, 256, (n_pages, 1, 16, x), generator=g, device="cuda", dtype=torch.uint8) for x in (32, 32, 2, 2)]
    want = [t.clone() for t in have]
    src, dst = torch.full((n,), -1, dtype=torch.int32, device="cuda"), torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for i, at in enumerate((0, 1, 2 ** 23 - 2, min(2 ** 23 - 1, n - 2), n // 2, n - 1)):
        src[at], dst[at] = i, 20 + i
    for a, b in zip(src[src >= 0].tolist(), dst[src >= 0].tolist()):  # (the second at a place is the one that is there)
        for t in want:
            t[b] = t[a]
    binding.fa_cache_copy(have[0], have[1], src, dst, k_scales=have[2], v_scales=have[3])
    for a, b in zip(have, want):
        assert torch.equal(a, b)


# rows, entries of a row, pages: beyond 16384 entries the table is renumbered by a launch of its own where the lists are in a workspace
@pytest.mark.parametrize("B,wide,n_pages", [(1, 16385, 5000), (3, 5463, 4097), (127, 129, 9001), (1025, 17, 4000), (7, 2341, 262145), (40, 411, 600001), (64, 257, 3000), (64, 256, 9001)])
@pytest.mark.parametrize("held", [False, True])
def test_large_tables_are_renumbered(B, wide, n_pages, held):
    g = np.random.default_rng(B + wide)
    table = g.integers(0, n_pages, (B, wide))
    table[g.random((B, wide)) < 0.7] = -1
    table = np.where(g.random((B, wide)) < 0.05, g.choice([-7, n_pages, 2 ** 31 - 1, -2 ** 31], (B, wide)), table)
    table[0, 0], table[-1, -1] = n_pages - 1, n_pages - 2
    keep = (g.random(n_pages) < 0.2) * g.choice([1, -4]) if held else None
    h = None if keep is None else _ints(keep)
    space = torch.empty(max(binding.fa_cache_pages_workspace_bytes(B, n_pages), 16), dtype=torch.uint8, device="cuda").random_(0, 256)
    for moves in (n_pages // 2, 1, 700, 0):
        want = pages_oracle.compact(table, keep, n_pages, moves or n_pages)
        if moves:
            _same(binding.fa_cache_compact(_ints(table), n_pages, moves=moves, held=h, workspace=space), want)
        else:  # in place, from a table whose entries are not aligned to 16 bytes
            t = torch.zeros(B * wide + 1, dtype=torch.int32, device="cuda")[1:].view(B, wide).copy_(_ints(table))
            got = binding.fa_cache_compact(t, n_pages, moves=n_pages, held=h, new_table=t, workspace=space)
            assert got[0] is t
            _same(got, want)


@pytest.mark.parametrize("B,B_new,wide,n_pages", [(3, 5, 513, 4000), (5, 9, 1025, 4096), (4, 40, 1025, 9000), (1024, 1100, 513, 600000), (1025, 700, 513, 600000), (2050, 1500, 3, 7000),
                                                  (1100, 1200, 1025, 300000)])
@pytest.mark.parametrize("held", [False, True])
def test_forks_of_wide_rows(B, B_new, wide, n_pages, held):
    """Lengths on both sides of entries 512 and 1024, free pages that only marks from there on decide about"""
    g = np.random.default_rng(B + wide)
    page = 16
    pool = g.permutation(n_pages)
    table = pool[g.integers(0, min(n_pages, 3 * wide), (B, wide))]
    table[:, :4] = -1
    table[0, 512:] = np.sort(pool)[:max(wide - 512, 0)]  # the lowest pages: taken by what lies behind entry 511 alone
    edges = [e * page + k for e in (511, 512, 513, 1023, 1024, 1025, wide - 1, wide) for k in (-1, 0, 1)]
    lens = g.choice([n for n in edges + [0, 5, wide * page // 2] if 0 <= n <= wide * page], B)
    lens[0] = wide * page
    parents = g.integers(0, B, B_new)
    parents[:3] = [0, B - 1, -1]
    keep = (g.random(n_pages) < 0.2) * g.choice([1, -4]) if held else None
    got = binding.fa_cache_fork(_ints(table), _ints(lens), _ints(parents), page, n_pages, held=None if keep is None else _ints(keep))
    _same(got, pages_oracle.fork(table, lens, parents, keep, page, n_pages))
