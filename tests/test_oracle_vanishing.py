"""The oracle's quantizer on rows so small that 127 / a is infinite: 0 stays 0, any other number is +-127."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("a", [3.6e-37, 2.0 ** -126, 1e-40, 2.0 ** -149])
def test_rows_below_the_range_of_the_factor(a):
    x = np.zeros((2, 64), np.float32)
    x[0, 1], x[0, 2], x[1, 5], x[1, 6] = a, -a, -a, -0.0
    q, s = oracle.quantize_tokenwise(x)
    assert q[0, 1] == 127 and q[0, 2] == -127 and q[1, 5] == -127
    assert np.count_nonzero(q) == 3
    assert np.array_equal(s, np.float32([a, a]) / np.float32(127))
