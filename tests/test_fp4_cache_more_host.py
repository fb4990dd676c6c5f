"""The 4-bit cache, as far as it goes without a GPU: what pins the oracle at the ends of the range."""
import numpy as np

from oracle import cache_oracle


def test_oracle_finite_elements_stay_finite():
    """Where the scale 2^126 would make 4 of it 2^128, it stays 2^125, and 6 of that stand for all from 5 2^125 on"""
    top = float(np.finfo(np.float32).max)
    x = np.zeros((5, 32), dtype=np.float32)
    x[0, :4] = [top, -top, 3.0e38, 3.38e38]
    x[1, :3] = [7 * 2.0 ** 125, 2.0 ** 125, -5.5 * 2.0 ** 125]
    x[2, :2] = np.nextafter(np.float32(7 * 2.0 ** 125), np.float32(np.inf)), 2.0 ** 125
    x[3, :2] = 7 * 2.0 ** 124, 2.0 ** 124
    x[4, :3] = top, np.inf, -np.inf
    codes, scales = cache_oracle.quantise_groups(x)
    assert scales[:, 0].tolist() == [252, 252, 252, 251, 252]
    back = cache_oracle.group_values(codes, scales)
    assert np.isfinite(back.astype(np.float32)).all()
    most = 6 * 2.0 ** 125
    np.testing.assert_array_equal(back[0, :4], [most, -most, most, most])
    np.testing.assert_array_equal(back[1, :3], [most, 2.0 ** 125, -most])
    np.testing.assert_array_equal(back[2, :2], [most, 2.0 ** 125])
    np.testing.assert_array_equal(back[3, :2], [6 * 2.0 ** 124, 2.0 ** 124])
    np.testing.assert_array_equal(back[4, :3], [most, most, -most])
