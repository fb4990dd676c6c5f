"""Pools and strides beyond 2^32 bytes and 2^31 elements: the calls give bit for bit what they give on small tensors of the same
contents.  (Every access is in a tensor that is as large as its strides say.)"""
import pytest
import torch

from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu


def _wide(t, batch_stride, head_stride):
    """t [B,H,N,d] in a tensor with these strides, in elements"""
    B, H, N, d = t.shape
    room = torch.empty(((B - 1) * batch_stride + (H - 1) * head_stride + N * d,), dtype=t.dtype, device="cuda")
    y = room.as_strided(t.shape, (batch_stride, head_stride, d, 1))
    y.copy_(t)
    return y


@pytest.mark.parametrize("cache,T,H", [("bf16", 1, 8), ("bf16", 20, 16), ("bf16", 20, 64), ("e4m3", 1, 16), ("e4m3", 5, 32), ("e4m3", 20, 64)])
def test_attention_over_a_pool_past_32_bits(cache, T, H):
    # 8 key/value heads: 1 to 160 rows of each; pages at both ends of the pool and in the middle
    H_kv, page, d, elem = 8, 1024, 256, 1 if cache == "e4m3" else 2
    n_pages = 2 ** 32 // (H_kv * page * d * elem) + 3
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [1, n_pages // 2, n_pages - 3]], dtype=torch.int32)
    small = torch.arange(6, dtype=torch.int32).view(2, 3)
    lens = torch.tensor([2 * page + 100, 2 * page - 3], dtype=torch.int32, device="cuda")
    q = inputs.normal_tensor(41, "q", (2, H, T, d), "bf16").cuda()
    big, little = {}, {}
    for x in ("k", "v"):
        values = inputs.normal_tensor(42, x, (6, H_kv, page, d), "bf16").cuda()
        if cache == "e4m3":
            values = values.float().clamp(-3, 3).to(torch.float8_e4m3fn).view(torch.uint8)
            scales = torch.rand((6, H_kv, page), generator=torch.Generator("cuda").manual_seed(1), device="cuda") + 0.1
            little[x + "_scales"], big[x + "_scales"] = scales, torch.zeros((n_pages, H_kv, page), device="cuda")
            big[x + "_scales"][table.flatten().cuda().long()] = scales
        little[x + "_pages"], big[x + "_pages"] = values, torch.zeros((n_pages, H_kv, page, d), dtype=values.dtype, device="cuda")
        for i, p in enumerate(table.flatten().tolist()):
            big[x + "_pages"][p] = values[i]
    for max_len in (0, 1 << 20):
        a = binding.fa_fwd_cache(q, block_table=table.cuda(), lens=lens, scale=0.06, max_len=max_len, **big)
        b = binding.fa_fwd_cache(q, block_table=small.cuda(), lens=lens, scale=0.06, max_len=max_len, **little)
        assert torch.isfinite(b[0]).all() and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("strides", [(2 ** 31 + 64, 4096), (4096 * 4, 2 ** 31 + 64)])
def test_strides_past_31_bits(strides):
    B, H, N, d, page = 2, 2, 3, 128, 16
    q, k, v = (inputs.normal_tensor(43, x, (B, H, N, d), "bf16").cuda() for x in ("q", "k", "v"))
    f, _ = binding.fa_rope_frequencies(d)
    # rotation: from and to, Q far and K near
    far = _wide(q, *strides)
    want = binding.fa_rope(q, f, k=k)
    got = binding.fa_rope(far, f, k=k, q_out=far)
    assert got[0] is far and torch.equal(far, want[0]) and torch.equal(got[1], want[1])
    far.copy_(q)
    table, lens = torch.arange(2 * 4, dtype=torch.int32, device="cuda").view(2, 4), torch.tensor([30, 5], dtype=torch.int32, device="cuda")
    pages = [[inputs.normal_tensor(44, x, (8, H, page, d), "bf16").cuda() for x in ("k", "v")] for _ in range(2)]
    # new tokens, queries and outputs
    binding.fa_cache_write(k, q, *pages[0], table, lens)
    binding.fa_cache_write(k, far, *pages[1], table, lens)
    assert torch.equal(pages[0][0], pages[1][0]) and torch.equal(pages[0][1], pages[1][1])
    o, lse = binding.fa_fwd_cache(q, *pages[0], table, lens, 0.1)
    got = binding.fa_fwd_cache(q, *pages[0], table, lens, 0.1, o=far)
    assert torch.equal(got[0], o) and torch.equal(got[1], lse)
    far.copy_(q)
    got = binding.fa_fwd_cache(far, *pages[0], table, lens, 0.1)
    assert torch.equal(got[0], o) and torch.equal(got[1], lse)
