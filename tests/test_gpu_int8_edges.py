"""GPU tests of the 8-bit projections where they can go wrong: the largest finite
values, and every form of their kernels that the rule takes at any size."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import int8
from linear_forms import CASES, form
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


@pytest.mark.parametrize("m,k,ns", CASES)
def test_linear_forms(api, m, k, ns):
    """y bit for bit on 400 channels (all of fewer), the first and last among them, on a
    workspace sized for the most rows and full of other bytes."""
    g = torch.Generator(device="cuda").manual_seed(m + k)
    w = torch.empty((m, k), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    some = torch.arange(m) if m <= 400 else torch.cat([torch.arange(150), torch.randint(150, m - 150, (100,)),
                                                       torch.arange(m - 150, m)])
    packed = torch.full((api.sb_linear_packed_bytes(m, k),), 0x55, dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(w, packed)
    wf = w[some.cuda()].float().cpu().numpy()
    del w
    ws = torch.full((api.sb_linear_workspace_bytes(m, k, 256),), 0xff, dtype=torch.uint8, device="cuda")
    for n in ns:
        say("linear", m, k, n, form(m, k, n))
        x = torch.empty((n, k), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        buf = torch.full((n * m + 64,), 7.0, device="cuda")
        y = buf[:n * m].view(n, m)
        api.sb_linear_quantized(packed, x, y, ws)
        torch.cuda.synchronize()
        assert (buf[n * m:] == 7.0).all()
        assert np.array_equal(y[:, some.cuda()].cpu().numpy(), int8.linear(x.float().cpu().numpy(), wf))


def test_linear_k_ranges_of_two_tiles_captured(api):
    """K ranges of 256 channels' groups and their join, replayed beside eager calls on a
    workspace of their own."""
    m, k, n = 8192, 28672, 100
    assert form(m, k, n) == ("ring", 2, 7, True)
    g = torch.Generator(device="cuda").manual_seed(6)
    packed = torch.empty(api.sb_linear_packed_bytes(m, k), dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(torch.empty((m, k), dtype=torch.bfloat16, device="cuda").normal_(generator=g), packed)
    x0 = torch.empty((n, k), device="cuda").normal_(generator=g)
    xd, y, y2 = x0.clone(), torch.zeros((n, m), device="cuda"), torch.zeros((n, m), device="cuda")
    ws, ws2 = (torch.empty(api.sb_linear_workspace_bytes(m, k, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.sb_linear_quantized(packed, xd, y, ws)
    for i in range(4):
        xd.copy_(x0 * (3.0 if i % 2 else -1.0) + i)
        y.zero_()
        graph.replay()
        api.sb_linear_quantized(packed, xd, y2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and y.abs().max() > 0
