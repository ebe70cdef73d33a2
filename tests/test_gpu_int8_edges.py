"""GPU tests of the 8-bit projections where they can go wrong: the largest finite
values."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import int8
from test_gpu_int8 import bf16, product

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    assert torch.cuda.is_available()
    return A


TOPS = [0x7f7f, 0x7f00, 0x7e02, 0x7e01, 0x7d93, 0x7180, 0x717f, 0x3f80, 0x0080]  # bfloat16 bits


def rows(g, k):
    """[len(TOPS)][k], the largest magnitude of each row one of TOPS, of either sign."""
    amax = (np.array(TOPS, np.uint32) << 16).view(np.float32)
    x = g.uniform(-1.0, 1.0, (len(TOPS), k)) * amax[:, None]
    x[:, 1] *= 1e-30
    x[:, k // 2], x[:, k - 1] = amax, -amax
    return bf16(x)


@pytest.mark.parametrize("size", [1.0, 2.0 ** -16])
@pytest.mark.parametrize("k", [40, 328, 1032])
def test_linear_largest_values(api, k, size):
    """Weight rows and token rows whose largest magnitude is up to the largest finite
    value, where 127 amax passes float32: y bit for bit.  Against operands of size 1 a y
    may pass float32 itself (|y| <= k amax size 4.5); against those of 2^-16 none does."""
    g = np.random.default_rng(k)
    plain = bf16(g.standard_normal((20, k)) * size)
    big = rows(g, k)
    f32 = big.float()
    f32[0, k - 1] = torch.finfo(torch.float32).max
    f32[1:, 2:] *= 1.0 - 2.0 ** -20 * torch.from_numpy(g.integers(0, 9, (len(TOPS) - 1, k - 2))).float()
    for what, w, x, dt in (("weights", big, plain, np.float64), ("bf16 rows", plain, big, np.float64),
                           ("f32 rows", plain, f32, np.float32)):
        say("linear, largest", what, k, size)
        got = product(api, w, x)
        with np.errstate(over="ignore"):
            ref = int8.linear(x.float().numpy(), w.float().numpy(), dt)
        assert np.array_equal(got, ref) and (size == 1.0 or np.isfinite(ref).all())
