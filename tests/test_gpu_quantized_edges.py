"""GPU tests of the 8-bit cache where it can go wrong: the largest finite values."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import quantized
from test_gpu_quantized import bf16, dev

pytestmark = pytest.mark.gpu

FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    assert torch.cuda.is_available()
    return A


# ---- blocks ------------------------------------------------------------------------

@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_quantize_largest_values(api, form, d):
    """Blocks whose largest magnitude is up to the largest bfloat16, where amax top
    passes float32: codes and scales bit for bit, neighbours in a word among them."""
    tops = [0x7f7f, 0x7f00, 0x7e80, 0x7e02, 0x7e01, 0x7d93, 0x7d92, 0x7d91, 0x7180, 0x717f, 0x0001, 0x0080]
    amax = (np.array(tops, np.uint32) << 16).view(np.float32).astype(np.float64)
    g = np.random.default_rng(d)
    x = g.uniform(-1.0, 1.0, (1, len(tops), 64, d)) * amax[None, :, None, None]
    x[..., 3] *= 1e-3
    x[..., 4] *= 1e-30
    x[:, :, 7, 5], x[:, :, 8, 5], x[:, :, 9, 6] = amax, -amax, amax
    x = bf16(x)
    assert np.array_equal(x.double().abs().amax((-2, -1)).numpy()[0], amax)
    cfg = api.attention_config(1, len(tops), len(tops), d)
    c = api.QuantizedKV(cfg, 64, 8, form)
    say("quantize the largest", form, d)
    api.sb_kv_quantize(cfg, dev(x), dev(x.transpose(2, 3)), 0, c, 0, 1)
    ko = torch.zeros((1, len(tops), 64, d), dtype=torch.bfloat16, device="cuda")
    vo = torch.zeros((1, len(tops), d, 64), dtype=torch.bfloat16, device="cuda")
    api.sb_kv_dequantize(cfg, c, 0, 1, ko, vo, 0)
    torch.cuda.synchronize()
    codes, s = quantized.quantize(x.double().numpy(), form)
    ref = bf16(codes.astype(np.float32) * s[..., None, None]).float().numpy().reshape(1, len(tops), 64, d)
    assert np.isfinite(ref).all() and np.abs(codes).max((-2, -1)).min() == quantized.TOP[form]
    for out, scale in ((ko, c.k_scale), (vo.transpose(2, 3), c.v_scale)):
        assert np.array_equal(scale.cpu().numpy(), s)
        assert np.array_equal(out.float().cpu().numpy(), ref)
