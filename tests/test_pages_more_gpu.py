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
