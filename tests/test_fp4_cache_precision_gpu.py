"""What attention over a 4-bit cache keeps of its operands, whatever the types and the number of rows: probabilities have 16 bits in their product
with V."""
import numpy as np
import pytest

from test_fp4_cache_gpu import Case
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
