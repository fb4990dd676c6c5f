"""How fa_fwd_cache divides its work: what a length that one sequence may have does to a large batch, and the workspace of either
division."""
import numpy as np
import pytest
import torch

from paper_2407_08608_amd import binding
from test_cache_host import P, _attend

# B, H, H_kv, T with 512 workgroups and more at whole sequences (256 of 17 to 64 rows)
_LARGE = [(64, 8, 8, 1), (64, 32, 8, 4), (512, 32, 8, 1), (32, 64, 8, 4), (32, 32, 8, 16), (32, 64, 8, 32)]
_CODES = [binding.FA_BF16, binding.FA_F16, binding.FA_FP8_E4M3]


@pytest.mark.parametrize("code", _CODES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,H_kv,T", _LARGE)
def test_a_long_sequence_in_a_large_batch_is_divided(B, H, H_kv, T, d, code):
    # a workgroup alone would take 65536 keys of one sequence while the others are done
    for max_len in (16384, 65536, 1 << 20):
        assert binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, max_len, code) > 0
    assert binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, 1000, code) == 0  # nothing to divide: one launch, no workspace


@pytest.mark.parametrize("H,H_kv,T,d,page,max_pages,code", [(4, 1, 1, 128, 64, 1024, binding.FA_BF16), (8, 8, 1, 64, 16, 4096, binding.FA_F16),
                                                            (16, 2, 33, 256, 16, 2048, binding.FA_FP8_E4M3)])
def test_a_divided_call_refuses_a_missing_small_or_misaligned_workspace(H, H_kv, T, d, page, max_pages, code):
    a = dict(B=1, H=H, H_kv=H_kv, T=T, d=d, page=page, max_pages=max_pages, tree=None, dense=binding.FA_F16 if code == binding.FA_F16 else binding.FA_BF16,
             cache=code)
    if code != binding.FA_FP8_E4M3:
        a.update(ks=None, vs=None)
    else:
        a.update(ks=P, vs=P)
    need = binding.fa_fwd_cache_workspace_bytes(1, H, H_kv, T, d, page * max_pages, code)
    assert need > 0
    assert _attend(**a, ws=None, ws_bytes=need) == 6 and _attend(**a, ws=P, ws_bytes=need - 1) == 6 and _attend(**a, ws=P + 8, ws_bytes=need) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cache,d,B,H,H_kv,T", [("bf16", "bf16", 128, 64, 8, 8, 1), ("f16", "e4m3", 64, 64, 16, 8, 2), ("bf16", "bf16", 64, 32, 32, 8, 5),
                                                      ("f16", "f16", 256, 64, 8, 8, 1), ("bf16", "e4m3", 128, 64, 16, 8, 33)])
def test_a_large_batch_with_one_long_sequence(dtype, cache, d, B, H, H_kv, T):
    from test_fwd_cache_gpu import Case, _random_tree

    g = np.random.default_rng(B + d)
    lens, counts, long = g.integers(0, 40, B), g.integers(0, min(T, 3) + 1, B), B // 3
    lens[long], counts[long] = 5003, T
    # a pool no larger than it has to be: pages where a sequence has tokens, none elsewhere
    pages = -(-(lens + T) // 16)
    table, at = np.full((B, max(pages)), -1, dtype=np.int32), 0
    for b in range(B):
        table[b, :pages[b]] = np.arange(at, at + pages[b])
        at += pages[b]
    c = Case(980 + d, dtype, cache, B, H, H_kv, T, d, 16, lens, counts, _random_tree(T, B, T) if T > 1 else None, width=-(-at // B), table=table)
    need = binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, 16 * table.shape[1], binding._CACHE_CODE[c.args["k_pages"].dtype])
    assert need > 0
    o, lse = c.run(workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    c.check(o, lse)
    there = torch.from_numpy(np.arange(T)[None, :] < c.counts[:, None]).cuda()[:, None].expand(B, H, T)
    again = c.run()
    assert torch.equal(again[0][there], o[there]) and torch.equal(again[1][there], lse[there])
    c.check(*c.run(max_len=100))  # the other division
