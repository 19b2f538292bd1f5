"""The plain form of the paged caches' codes at the ends of the types' ranges."""
import numpy as np

from oracle import paged_oracle as G


def test_finite_rows_stay_finite():
    """Every row widens within fp32 and bf16 (largest number 255 2^120), the nearest code where there is one."""
    bf16_max = 255 * 2.0 ** 120
    for top in (1.75 * 2.0 ** 127, 1.76 * 2.0 ** 127, 1.9 * 2.0 ** 127, 248 * 2.0 ** 120, 3.38e38, bf16_max,
                float(np.finfo(np.float32).max)):
        for sign in (1.0, -1.0):
            row = np.array([sign * top, np.inf, -np.inf, 0.0, 1.0])
            x = G.widen(*G.quantise(row))
            assert np.all(np.abs(x) <= bf16_max)
            assert abs(x[0] - sign * top) <= 2.0 ** -4 * top
            assert x[1] >= abs(x[0]) and x[2] == -x[1]
    # unchanged below: 448 2^119
    x = G.widen(*G.quantise(np.array([448 * 2.0 ** 119, 100 * 2.0 ** 119])))
    assert x[0] == 448 * 2.0 ** 119 and x[1] in (96 * 2.0 ** 119, 104 * 2.0 ** 119)
