"""CPU pins of the 8-bit projections' oracle at the largest finite values."""
import numpy as np
import pytest

from oracle import int8


@pytest.mark.parametrize("dt", [np.float32, np.float64])
def test_codes_do_not_depend_on_a_power_of_two(dt):
    """x and 2^e x have the same codes, up to the largest finite float32."""
    g = np.random.default_rng(0)
    x = g.uniform(-1.0, 1.0, (6, 200)).astype(np.float32)
    x[:, 7] = 1.0 - 2.0 ** -24
    codes, scale = int8.quantize(x, dt)
    assert np.abs(codes).max() == 127
    for e in (50, 99, 100, 101, 121, 122, 127, 128):
        big, s = int8.quantize(np.ldexp(x, e), dt)
        assert np.array_equal(big, codes) and np.array_equal(s, np.ldexp(scale, e))
