"""The 4-bit cache at the ends of the range: finite elements are finite when they come back."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle
from paper_2407_08608_amd import binding

pytestmark = pytest.mark.gpu

_T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dense", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_finite_elements_stay_finite(dense, d):
    B, H_kv, T, page, dt = 2, 2, 40, 16, _T[dense]
    g = torch.Generator(device="cuda").manual_seed(d)
    # exponents of the largest magnitude up to the type's last, and infinities among the largest numbers
    x = [(torch.rand((B, H_kv, T, d), generator=g, device="cuda", dtype=torch.float64) * 2 - 1) * 2.0 ** torch.randint(123, 129, (B, H_kv, T, d // 32), generator=g, device="cuda")
         .repeat_interleave(32, -1) for _ in range(2)]
    k, v = (y.clamp(-torch.finfo(dt).max, torch.finfo(dt).max).to(dt) for y in x)
    k[0, 0, 0, :2], k[0, 0, 1, 32:34] = torch.finfo(dt).max, torch.finfo(dt).min
    v[1, 1, 3, 5], v[1, 1, 3, 6] = float("inf"), float("-inf")
    pages, scales = ([torch.zeros((8, H_kv, page, n), dtype=torch.uint8, device="cuda") for _ in range(2)] for n in (d // 2, d // 32))
    table = torch.tensor([[3, 1, 7], [0, 6, 2]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    binding.fa_cache_write(k, v, pages[0], pages[1], table, lens, k_scales=scales[0], v_scales=scales[1])
    for out in (torch.float32, torch.bfloat16):
        got = binding.fa_cache_read(pages[0], pages[1], table, lens + T, N=T, dtype=out, k_scales=scales[0], v_scales=scales[1])
        for y, given in zip(got, (k, v)):
            assert y.isfinite().all()
            want = cache_oracle.group_values(*cache_oracle.quantise_groups(given.float().cpu().numpy()))
            np.testing.assert_array_equal(y.double().cpu().numpy(), want)  # (a bf16 number, whatever the type)
