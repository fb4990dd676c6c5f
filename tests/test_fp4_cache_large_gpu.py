"""4-bit pools beyond 2^32 bytes: written, read and attended over, bit for bit as small ones of the same contents."""
import pytest
import torch

from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu

_H_KV, _PAGE, _D = 8, 1024, 256
_N_PAGES = 2 ** 32 // (_H_KV * _PAGE * _D // 2) + 3


@pytest.fixture(scope="module")
def pools():
    """(table, pages and scales) of the large pool, and of a small one; pages at both ends of the large one and in its middle"""
    table = torch.tensor([[_N_PAGES - 1, 0, _N_PAGES - 2], [1, _N_PAGES // 2, _N_PAGES - 3]], dtype=torch.int32)
    g = torch.Generator("cuda").manual_seed(3)
    big, little = {}, {}
    for x in ("k", "v"):
        for n, last, lo, hi in (("_pages", _D // 2, 0, 256), ("_scales", _D // 32, 123, 128)):
            little[x + n] = torch.randint(lo, hi, (6, _H_KV, _PAGE, last), generator=g, device="cuda", dtype=torch.uint8)
            big[x + n] = torch.zeros((_N_PAGES, _H_KV, _PAGE, last), device="cuda", dtype=torch.uint8)
            for i, p in enumerate(table.flatten().tolist()):
                big[x + n][p] = little[x + n][i]
    return (dict(big, block_table=table.cuda()), dict(little, block_table=torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,H", [(1, 8), (3, 16), (20, 16), (20, 64)])
def test_attention(pools, dtype, T, H):
    q = inputs.normal_tensor(41, "q", (2, H, T, _D), dtype).cuda()
    lens = torch.tensor([2 * _PAGE + 100, 2 * _PAGE - 3], dtype=torch.int32, device="cuda")
    for max_len in (0, 1 << 20):
        got, want = (binding.fa_fwd_cache(q, lens=lens, scale=_D ** -0.5, max_len=max_len, **x) for x in pools)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.isfinite(want[0]).all()


def test_writing_and_reading(pools):
    k, v = (inputs.normal_tensor(43, n, (2, _H_KV, 50, _D), "bf16").cuda() for n in "kv")
    lens = torch.tensor([2 * _PAGE - 20, 2 * _PAGE], dtype=torch.int32, device="cuda")
    out = []
    for x in pools:
        pages, table = [x["k_pages"], x["v_pages"]], x["block_table"]
        scales = dict(k_scales=x["k_scales"], v_scales=x["v_scales"])
        binding.fa_cache_write(k, v, *pages, table, lens, **scales)
        read = [torch.zeros((2, _H_KV, 3 * _PAGE, _D), device="cuda", dtype=torch.bfloat16) for _ in "kv"]
        binding.fa_cache_read(*pages, table, lens + 50, k=read[0], v=read[1], **scales)
        out.append((read, [x[n][table.flatten().long()] for n in ("k_pages", "v_pages", "k_scales", "v_scales")]))
    for a, b in zip(*(r + p for r, p in out)):
        assert torch.equal(a, b) and (a != 0).any()
