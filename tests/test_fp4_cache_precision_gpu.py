"""What attention over a 4-bit cache keeps of its operands, whatever the types and the number of rows: probabilities have 16 bits in their product
with V, and a product of Q and K is exact, however far a row's scales are apart.

The bounds are those of Case: e_s = (2 d + 4) 2^-24 scale max_j sum |q k_j| holds for fp16 Q as two bf16 numbers h + r too.  That is exact, so are 2 d products,
and their sum is off by 2 d 2^-24 sum (|h k| + |r k|) at most, where |h| + |r| <= (1 + 2^-7) |q|: 2 d 2^-7 <= 4 up to d = 256."""
import numpy as np
import pytest
import torch

from test_fp4_cache_gpu import Case, _FORMS
from test_fwd_cache_gpu import _random_tree

pytestmark = pytest.mark.gpu


# rows to a key/value head: 17 to 32, 33 to 64, and more
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 2, 5), (64, 8, 2, 12), (64, 8, 2, 40), (128, 8, 2, 5), (128, 8, 2, 12), (128, 8, 2, 40), (256, 8, 2, 5), (256, 8, 2, 12),
                                        (256, 4, 1, 40)])
@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_probabilities_have_16_bits_with_many_rows(d, H, H_kv, T, max_len):
    """The bound of few rows, eps_p = 2^-16, which probabilities as one bf16 number (2^-8) do not keep: columns of V whose weighted mean is next
    to zero, some among thousands of random ones, show their rounding and little of the output's."""
    c = Case(800 + T + d, "bf16", 2, H, H_kv, T, d, 16, [150, 333], tree=_random_tree(T, 2, T))
    c.rows = 16
    c.check(*c.run(max_len=max_len))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_a_large_group_that_meets_zeros(dtype, d, H, H_kv, T, max_len):
    """One group of each key has a scale 2^40 times and more the others', and Q zeros there: the score is that of the others"""
    c = Case(900 + T + d, dtype, 2, H, H_kv, T, d, 16, [150, 70], tree=_random_tree(T, 2, T))
    scales = c.host["k_scales"]
    scales[..., 1] = np.where(scales[..., 1] == 255, 255, np.minimum(scales[..., 1].astype(int) + 44, 254))
    c.args["k_scales"] = torch.from_numpy(scales).cuda()
    c.q[..., 32:64] = 0
    c.check(*c.run(max_len=max_len))


@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
def test_the_smallest_and_largest_queries(d, H, H_kv, T):
    # multiples of fp16's smallest number, most of them subnormal, and numbers up to its largest, in groups whose keys make up for it
    c = Case(950 + T + d, "f16", 2, H, H_kv, T, d, 16, [150, 70], tree=_random_tree(T, 2, T))
    g = np.random.default_rng(T)
    q = g.standard_normal(c.q.shape)
    q[..., :32] = np.round(q[..., :32] * 300) * 2.0 ** -24
    q[..., 32:] = np.clip(q[..., 32:] * 30000, -65504, 65504)
    c.q = torch.from_numpy(q).to(torch.float16)
    for n, by in ((slice(0, 1), 15), (slice(1, None), -15)):
        s = c.host["k_scales"][..., n]
        c.host["k_scales"][..., n] = np.where(s == 255, 255, s.astype(int) + by)
    c.args["k_scales"] = torch.from_numpy(c.host["k_scales"]).cuda()
    c.check(*c.run())
    assert len(c.q[c.q.abs() < 2.0 ** -14].unique()) > 100  # (subnormal ones)
