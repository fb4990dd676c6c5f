"""fa_cache_fork, fa_cache_extend, fa_cache_compact and fa_cache_copy: exactly what the oracle gives, whatever the tables hold."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle
from paper_2407_08608_amd import binding

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int64), dtype=torch.int32, device="cuda")


def _tables(seed, B, wide, page, n_pages, shared=0.3, bad=0.1):
    """Random rows: own pages, some of other rows' (shared prefixes and not), some that are none; lengths from negative to past the table"""
    g = np.random.default_rng(seed)
    table = g.integers(0, n_pages, (B, wide))
    for b in range(1, B):
        if g.random() < shared:
            table[b, :g.integers(0, wide + 1)] = table[g.integers(0, b), 0]
        if g.random() < shared:
            n = g.integers(0, wide + 1)
            table[b, :n] = table[g.integers(0, b), :n]
    table = np.where(g.random((B, wide)) < bad, g.choice([-1, -7, n_pages, 2 ** 31 - 1, -2 ** 31], (B, wide)), table)
    lens = g.integers(0, wide * page + 1, B)
    lens[g.random(B) < 0.2] = g.choice([0, -3, 2 ** 31 - 1, wide * page, page])
    return g, table.astype(np.int64), lens


def _same(got, want):
    assert len(got) == len(want)
    for i, (a, b) in enumerate(zip(got, want)):
        np.testing.assert_array_equal(a.cpu().numpy(), np.asarray(b).reshape(tuple(a.shape)), err_msg=str(i))


# rows, new rows, width, page, pages of the pool
_SIZES = [(1025, 3, 2, 16, 4000), (5, 1025, 4, 16, 4096), (30, 40, 150, 16, 4097), (1, 1, 1, 16, 1), (1, 1, 1, 16, 2), (2, 5, 3, 16, 40), (4, 16, 7, 1, 100), (16, 16, 20, 16, 700), (7, 3, 33, 48, 300), (64, 64, 9, 16, 601),
          (3, 1500, 2, 16, 4000), (1030, 1025, 3, 5, 5000), (5, 9, 300, 64, 1100)]


@pytest.mark.parametrize("B,B_new,wide,page,n_pages", _SIZES)
@pytest.mark.parametrize("held", [False, True])
def test_fork(B, B_new, wide, page, n_pages, held):
    for seed in range(4):
        g, table, lens = _tables(seed, B, wide, page, n_pages, bad=0.1 if seed else 0.0)
        parents = g.integers(0, B, B_new)
        parents[g.random(B_new) < 0.1] = g.choice([-1, B, -2 ** 31])
        keep = (g.random(n_pages) < 0.2) * g.choice([1, -4]) if held else None
        got = binding.fa_cache_fork(_ints(table), _ints(lens), _ints(parents), page, n_pages, held=None if keep is None else _ints(keep))
        _same(got, pages_oracle.fork(table, lens, parents, keep, page, n_pages))


@pytest.mark.parametrize("B,B_new,wide,page,n_pages", _SIZES)
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("T", [1, 40])
def test_extend(B, B_new, wide, page, n_pages, held, T):
    for seed in range(4):
        g, table, lens = _tables(seed, B, wide, page, n_pages, bad=0.5 if seed else 1.0)
        counts = None if seed == 3 else g.integers(-2, T + 3, B)
        keep = (g.random(n_pages) < 0.2) * g.choice([1, -4]) if held else None
        if seed == 2:
            table[:, -(wide // 2):] = -1
        t = _ints(table)
        got = binding.fa_cache_extend(t, _ints(lens), T, page, n_pages, counts=None if counts is None else _ints(counts), held=None if keep is None else _ints(keep))
        assert got[0] is t
        n = np.full(B, T) if counts is None else np.minimum(counts, T)
        want = pages_oracle.extend(table, lens, n, keep, page, n_pages)
        _same(got, want)
        again = binding.fa_cache_extend(t, _ints(lens), T, page, n_pages, counts=None if counts is None else _ints(counts), held=None if keep is None else _ints(keep))
        _same(again, (want[0], want[1]))  # (what was not there is still missing)


@pytest.mark.parametrize("B,wide,page,n_pages,T", [(1, 8200, 16, 8200, 131072), (3, 2100, 16, 4096, 20000), (1100, 70, 16, 9000, 100), (1, 1025, 1, 1030, 1024),
                                                   (2, 1030, 1, 2100, 1030), (2050, 4, 16, 9000, 16)])
def test_extend_by_prompts(B, wide, page, n_pages, T):
    """Many entries of few sequences, between sequences that get one, none, or have their pages"""
    g = np.random.default_rng(B)
    table = np.full((B, wide), -1)
    lens = g.integers(0, 4 * page, B)
    for b in range(B):
        table[b, :lens[b] // page + 1] = g.integers(0, n_pages // 2, lens[b] // page + 1)
    table[g.random((B, wide)) < 0.05] = n_pages - 1
    for counts in (None, np.where(g.random(B) < 0.5, g.integers(0, 3, B), T)):
        want = pages_oracle.extend(table, lens, np.full(B, T) if counts is None else counts, None, page, n_pages)
        got = binding.fa_cache_extend(_ints(table), _ints(lens), T, page, n_pages, counts=None if counts is None else _ints(counts))
        _same(got, want)


def test_extend_past_the_table():
    """All of a sequence's places, and some, are past it; the others get theirs"""
    table = np.full((3, 4), -1)
    for lens in ([64, 0, 10], [60, 2 ** 31 - 1, 63], [64, 64, 100]):
        for T in (1, 16, 100):
            _same(binding.fa_cache_extend(_ints(table), _ints(lens), T, 16, 20), pages_oracle.extend(table, lens, [T] * 3, None, 16, 20))


@pytest.mark.parametrize("B,B_new,wide,page,n_pages", _SIZES)
@pytest.mark.parametrize("held", [False, True])
def test_compact(B, B_new, wide, page, n_pages, held):
    for seed in range(4):
        g, table, _ = _tables(seed, B, wide, page, n_pages, bad=(0.1, 0.9, 0.5, 1.0)[seed])
        keep = (g.random(n_pages) < 0.2) * g.choice([1, -4]) if held else None
        k = None if keep is None else _ints(keep)
        for moves in (None, 1, 3, 2 * n_pages + 5):
            got = binding.fa_cache_compact(_ints(table), n_pages, moves=moves, held=k)
            n = max(n_pages // 2, 1) if moves is None else moves
            _same(got, pages_oracle.compact(table, keep, n_pages, n))
        t = _ints(table)
        assert binding.fa_cache_compact(t, n_pages, held=k, new_table=t)[0] is t  # in place
        _same((t,), pages_oracle.compact(table, keep, n_pages, n_pages)[:1])


@pytest.mark.parametrize("n_pages", [262144, 262145, 600001])
def test_pools_of_more_pages_than_are_looked_at_at_a_time(n_pages):
    g = np.random.default_rng(n_pages)
    B, wide, page = 40, 50, 16
    table = g.integers(0, n_pages, (B, wide))
    table[0, :8] = [0, 262143, n_pages - 1, 262142, 31, 32, n_pages - 2, 100]
    lens = g.integers(0, wide * page - 20, B)
    keep = np.zeros(n_pages, dtype=np.int64)
    keep[:262144 - 10] = 1  # free pages on both sides of the border
    keep[n_pages - 1] = 1
    parents = g.integers(0, B // 2, B)
    for held in (None, keep):
        h = None if held is None else _ints(held)
        _same(binding.fa_cache_fork(_ints(table), _ints(lens), _ints(parents), page, n_pages, held=h), pages_oracle.fork(table, lens, parents, held, page, n_pages))
        bare = np.where(np.arange(wide) < (lens // page)[:, None], table, -1)
        _same(binding.fa_cache_extend(_ints(bare), _ints(lens), 20, page, n_pages, held=h), pages_oracle.extend(bare, lens, [20] * B, held, page, n_pages))
        _same(binding.fa_cache_compact(_ints(table), n_pages, held=h, moves=3000), pages_oracle.compact(table, held, n_pages, 3000))


def _cache(seed, kind, n_pages, H_kv, page, d):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind in ("bf16", "f16"):
        return [torch.randn((n_pages, H_kv, page, d), generator=g, device="cuda").to(torch.bfloat16 if kind == "bf16" else torch.float16) for _ in range(2)] + [None, None]
    last, group = (d, ()) if kind == "e4m3" else (d // 2, (d // 32,))
    pages = [torch.randint(0, 256, (n_pages, H_kv, page, last), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    if kind == "e4m3":
        return pages + [torch.rand((n_pages, H_kv, page), generator=g, device="cuda") for _ in range(2)]
    return pages + [torch.randint(0, 256, (n_pages, H_kv, page) + group, generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3", "4bit"])
@pytest.mark.parametrize("H_kv,page,d", [(1, 16, 64), (2, 16, 128), (3, 48, 256), (8, 128, 128), (5, 16, 64)])
def test_copy(kind, H_kv, page, d):
    n_pages = 60
    have = _cache(H_kv + d, kind, n_pages, H_kv, page, d)
    order = np.random.default_rng(d).permutation(n_pages)
    src, dst = order[:20].copy(), order[20:40].copy()
    src[3], dst[4], src[5], dst[6], src[7] = -1, -1, n_pages, 2 ** 31 - 1, -2 ** 31
    dst[8] = src[8]
    src[9] = src[10]  # one page to two places
    want = [None if t is None else t.clone() for t in have]
    for a, b in zip(src.tolist(), dst.tolist()):
        if 0 <= a < n_pages and 0 <= b < n_pages:
            for t in want:
                if t is not None:
                    t[b] = t[a].clone()
    got = binding.fa_cache_copy(have[0], have[1], _ints(src), _ints(dst), k_scales=have[2], v_scales=have[3])
    assert got[0] is have[0] and got[1] is have[1]
    for a, b in zip(have, want):
        assert a is None or torch.equal(a, b)


def test_copies_of_pages_past_32_bits():
    # 5 GiB of K: pages whose bytes lie past 2^32
    n_pages, H_kv, page, d = 10240, 8, 128, 256
    k = torch.empty((n_pages, H_kv, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for t, x in ((k, 1.0), (v, 2.0)):
        t[10239], t[0], t[1], t[5000] = x, -x, 3 * x, 0.0
    binding.fa_cache_copy(k, v, _ints([10239, 0]), _ints([1, 10238]))
    for t, x in ((k, 1.0), (v, 2.0)):
        assert (t[1] == x).all() and (t[10238] == -x).all() and (t[10239] == x).all() and (t[0] == -x).all() and (t[5000] == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "4bit"])
def test_a_beam_search_keeps_what_its_sequences_hold(kind):
    """Forks, copies, extensions, writes and compactions in turn, in a pool that is just large enough: what a sequence holds, read back
    through the cache, is what a list of its own tokens says"""
    H_kv, page, d, beams, wide = 2, 16, 64, 6, 9
    n_pages = 40
    cache = [_cache(i, kind, n_pages, H_kv, page, d) for i in range(2)]  # two layers
    g = np.random.default_rng(9)
    gen = torch.Generator(device="cuda").manual_seed(1)
    table, lens = _ints(np.full((beams, wide), -1)), _ints([0] * beams)
    said = [[torch.zeros((2, H_kv, 0, d), device="cuda") for _ in range(beams)] for _ in range(2)]
    for step in range(30):
        T = int(g.integers(1, 6))
        counts = g.integers(0, T + 1, beams)
        table, missing = binding.fa_cache_extend(table, lens, T, page, n_pages, counts=_ints(counts))
        assert missing.item() == 0
        for layer, (kp, vp, ks, vs) in enumerate(cache):
            # (values that a 4-bit group holds exactly)
            new = [torch.randint(-2, 3, (beams, H_kv, T, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
            binding.fa_cache_write(new[0], new[1], kp, vp, table, lens, counts=_ints(counts), k_scales=ks, v_scales=vs)
            for b in range(beams):
                said[layer][b] = torch.cat((said[layer][b], torch.stack([x[b, :, :counts[b]].float() for x in new])), 2)
        lens = lens + _ints(counts)
        parents = g.integers(0, beams, beams) if step % 4 else g.permutation(beams)
        if step % 7 == 6:
            parents[g.integers(0, beams)] = -1
        if max(lens.tolist()) > wide * page - 12:
            parents[:] = np.where(np.isin(parents, np.nonzero(lens.cpu().numpy() > wide * page - 12)[0]), -1, parents)
        table, lens, src, dst, missing = binding.fa_cache_fork(table, lens, _ints(parents), page, n_pages)
        assert missing.item() == 0
        moves = [(src, dst)]
        if step % 3 == 2:
            table, src, dst, top = binding.fa_cache_compact(table, n_pages)
            moves.append((src, dst))
            assert top.item() == len({p for p in table.flatten().tolist() if p >= 0})
        for kp, vp, ks, vs in cache:
            for src, dst in moves:
                binding.fa_cache_copy(kp, vp, src, dst, k_scales=ks, v_scales=vs)
        for layer, (kp, vp, ks, vs) in enumerate(cache):
            said[layer] = [said[layer][p] if p >= 0 else torch.zeros((2, H_kv, 0, d), device="cuda") for p in parents]
            read = binding.fa_cache_read(kp, vp, table, lens, N=wide * page, k_scales=ks, v_scales=vs)
            for b in range(beams):
                assert lens[b].item() == said[layer][b].shape[2]
                for i in range(2):
                    assert torch.equal(read[i][b, :, :lens[b].item()].float(), said[layer][b][i]), (step, layer, b)


def test_replayed_steps_and_another_stream():
    """Fork, copy and extend captured once: every replay, on new parents and lengths, gives what the calls give"""
    B, wide, page, n_pages = 8, 12, 16, 130
    kp, vp, _, _ = _cache(3, "bf16", n_pages, 2, page, 64)
    g = np.random.default_rng(4)
    own = g.permutation(n_pages)[:B * wide].reshape(B, wide)
    table, lens, parents = _ints(own), _ints([0] * B), _ints([0] * B)
    out = [_ints(np.zeros(s)) for s in ((B, wide), B, B, B, 1, 1)]
    space = torch.empty(max(binding.fa_cache_pages_workspace_bytes(B, n_pages), 16), dtype=torch.uint8, device="cuda")

    def step():
        binding.fa_cache_fork(table, lens, parents, page, n_pages, new_table=out[0], new_lens=out[1], src=out[2], dst=out[3], missing=out[4], workspace=space)
        binding.fa_cache_copy(kp, vp, out[2], out[3])
        binding.fa_cache_extend(out[0], out[1], 3, page, n_pages, missing=out[5], workspace=space)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        n, p = g.integers(0, wide * page - 3, B), g.integers(-1, B, B)
        lens.copy_(_ints(n))
        parents.copy_(_ints(p))
        before = [kp.clone(), vp.clone()]
        if replay % 2:
            graph.replay()
        else:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        rows, new_lens, src, dst, missing = pages_oracle.fork(own, n, p, None, page, n_pages)
        rows, none = pages_oracle.extend(rows, new_lens, [3] * B, None, page, n_pages)
        _same(out, (rows, new_lens, src, dst, missing, none))
        for a, b in zip(src, dst):
            if a >= 0:
                for t in before:
                    t[b] = t[a]
        assert torch.equal(kp, before[0]) and torch.equal(vp, before[1])


def test_the_binding_refuses_what_does_not_fit():
    t, lens, p = _ints(np.zeros((3, 4))), _ints([1, 2, 3]), _ints([0, 1])
    fork = lambda *a, **kw: binding.fa_cache_fork(*a, **kw)  # noqa: E731
    small = torch.empty((64,), dtype=torch.uint8, device="cuda")
    for call, kind in ((lambda: fork(t.long(), lens, p, 16, 9), ValueError), (lambda: fork(t, lens[:2], p, 16, 9), ValueError),
                       (lambda: fork(t, lens, p[None], 16, 9), ValueError), (lambda: fork(t, lens, p.cpu(), 16, 9), ValueError),
                       (lambda: fork(t, lens, p, 0, 9), binding.FaError), (lambda: fork(t, lens, p, 16, 0), binding.FaError),
                       (lambda: fork(t, lens, p, 16, 9, held=lens), ValueError), (lambda: fork(t, lens, p, 16, 5000, workspace=small), binding.FaError),
                       (lambda: fork(t, lens, _ints([0, 1, 2]), 16, 9, new_table=t), binding.FaError),
                       (lambda: fork(t, lens, _ints([0, 1, 2]), 16, 9, new_lens=lens), binding.FaError),
                       (lambda: fork(t, lens, p[:0], 16, 9), binding.FaError), (lambda: fork(t, lens, p, 16, 9, src=lens), ValueError),
                       (lambda: binding.fa_cache_extend(t, lens, 0, 16, 9), binding.FaError), (lambda: binding.fa_cache_extend(t, lens, 1, 16, 9, counts=p), ValueError),
                       (lambda: binding.fa_cache_extend(t.t(), lens, 1, 16, 9), ValueError), (lambda: binding.fa_cache_extend(t, lens, 2 ** 31 - 1, 16, 9), binding.FaError),
                       (lambda: binding.fa_cache_compact(t, 9, moves=0), binding.FaError), (lambda: binding.fa_cache_compact(t, 9, moves=4, src=lens), ValueError),
                       (lambda: binding.fa_cache_compact(t, 0), binding.FaError), (lambda: binding.fa_cache_compact(t[0], 9), ValueError)):
        with pytest.raises(kind):
            call()
    k = torch.zeros((4, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    c, s4, s8 = k[..., :32].to(torch.uint8).contiguous(), torch.zeros((4, 1, 16, 2), dtype=torch.uint8, device="cuda"), torch.ones((4, 1, 16), device="cuda")
    copy = binding.fa_cache_copy
    for call, kind in ((lambda: copy(k, k[:3], p, p), ValueError), (lambda: copy(k, k, p, lens), ValueError), (lambda: copy(k, k, p[:0], p[:0]), binding.FaError),
                       (lambda: copy(c, c, p, p, k_scales=s4, v_scales=s8), ValueError), (lambda: copy(c, c, p, p, k_scales=s4[..., :1], v_scales=s4), ValueError),
                       (lambda: copy(c, c, p, p), ValueError), (lambda: copy(c, c, p, p, k_scales=s8, v_scales=s8), binding.FaError),
                       (lambda: copy(k, k, p, p, k_scales=s8, v_scales=s8), ValueError), (lambda: copy(k.float(), k.float(), p, p), ValueError)):
        with pytest.raises(kind):
            call()
