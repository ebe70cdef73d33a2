"""CPU pins of the 8-bit projections' oracle, and the host checks of their
entry points (nothing here launches)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import decoder, int8
from paper_2506_01979_amd import synth


def test_linear_is_the_product_to_half_a_code():
    """Every code is within half a step of its value, so y is within
    amax_x / 254 |w|_1 + amax_w / 254 (|x|_1 + K amax_x / 254) of x W^T."""
    g = np.random.default_rng(0)
    x, w = g.standard_normal((5, 300)), g.standard_normal((7, 300))
    y = int8.linear(x, w)
    sx, sw = np.abs(x).max(-1)[:, None] / 254, np.abs(w).max(-1)[None] / 254
    bound = sx * np.abs(w).sum(-1)[None] + sw * (np.abs(x).sum(-1)[:, None] + 300 * sx)
    assert np.all(np.abs(y - x @ w.T) <= bound * (1 + 1e-5))
    codes, scale = int8.quantize(x)
    assert np.abs(codes).max() == 127 and np.all(np.abs(codes * scale[:, None] - x) <= sx * (1 + 1e-5))


def test_special_rows():
    x = np.ones((4, 8))
    x[0] = 0
    x[1, 3] = np.nan
    x[2, 1] = np.inf
    codes, scale = int8.quantize(x)
    assert scale[0] == 0 and np.isnan(scale[1]) and np.isnan(scale[2]) and scale[3] == np.float32(1 / 127)
    assert np.all(codes[:3] == 0) and np.all(codes[3] == 127)
    assert np.array_equal(int8.quantize(np.array([[254.0, 1.0, 3.0, -5.0]]))[0], [[127, 0, 2, -2]])   # ties to even


@pytest.mark.parametrize("sname", ["tiny", "small_gqa_bf16"])
def test_forward_without_quantisation_is_the_decoder(sname):
    shape = synth.SHAPES[sname]
    W = synth.model_weights(shape)
    g = np.random.default_rng(1)
    K, V = (g.standard_normal((shape.n_layers, shape.n_kv_heads, 9, shape.head_dim)) for _ in range(2))
    parents, tokens = [-1, 0, 0, 2, 1], g.integers(0, shape.vocab, 5)
    ref, kr, vr = decoder.tree_forward(shape, W, K, V, 9, tokens, parents, "f64")
    out, k, v = int8.tree_forward(shape, W, K, V, 9, tokens, parents, project=lambda x, w: x @ w.astype(np.float64).T,
                                  store=lambda x: x)
    assert np.allclose(out, ref, rtol=1e-9, atol=1e-12)
    assert np.allclose(k, kr, rtol=1e-9, atol=1e-12) and np.allclose(v, vr, rtol=1e-9, atol=1e-12)


def test_forward_is_near_the_decoder():
    """8 bits a token and channel: a percent or two of the logits' size."""
    shape = synth.SHAPES["small_bf16"]
    W = synth.model_weights(shape)
    parents, tokens = [-1, 0, 0, 2], np.array([3, 999, 4, 5])
    ref, _, _ = decoder.tree_forward(shape, W, [None] * 2, [None] * 2, 0, tokens, parents, "f64")
    out, _, _ = int8.tree_forward(shape, W, [None] * 2, [None] * 2, 0, tokens, parents)
    rel = np.linalg.norm(out - ref) / np.linalg.norm(ref)
    assert 1e-4 < rel < 0.1


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    return A


def test_linear_refusals(api):
    assert api.sb_linear_packed_bytes(100, 65) == 7 * 4 * 1024 + 7 * 64     # 7 tiles, 4 k-steps, scales
    for m, k in ((0, 8), (8, 0), (8, 32769), ((1 << 24) + 1, 8), (-1, 8)):
        assert api.sb_linear_packed_bytes(m, k) == 0 and api.sb_linear_workspace_bytes(m, k, 1) == 0
        assert api.lib.sb_linear_pack(m, k, 16, 16, None) == 1
    assert api.lib.sb_linear_pack(8, 8, None, 16, None) == 1 and api.lib.sb_linear_pack(8, 8, 16, None, None) == 1
    assert api.lib.sb_linear_pack(8, 8, 16, 24, None) == 1
    sizes = [api.sb_linear_workspace_bytes(100, 4096, n) for n in range(1, 257)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert api.sb_linear_workspace_bytes(8, 8, 0) == 0 and api.sb_linear_workspace_bytes(8, 8, 257) == 0
    need = api.sb_linear_workspace_bytes(100, 65, 3)

    def call(m=100, k=65, w=16, n=3, x=16, dt=api.SB_BF16, y=16, ws=16, size=need):
        return api.lib.sb_linear_quantized(m, k, w, n, x, dt, y, ws, size, None)
    assert call(m=0) == 1 and call(k=32769) == 1 and call(n=0) == 1 and call(n=257) == 1
    for f in ("w", "x", "y", "ws"):
        assert call(**{f: None}) == 1
    assert call(w=24) == 1 and call(ws=24) == 1
    assert call(dt=api.SB_INT8) == 4 and call(dt=7) == 4 and call(size=need - 1) == 3


def test_int8_model_host_side(api):
    shape = synth.SHAPES["llama7b"]
    c = api.make_config(shape, "int8")
    assert api.sb_packed_bytes(c, api.SB_W_QKV) == 12288 * 4096 + 12288 * 4
    assert api.sb_packed_bytes(c, api.SB_W_GATE_UP) == 22016 * 4096 + 22016 * 4
    assert api.sb_packed_bytes(c, api.SB_W_DOWN) == 4096 * 11008 + 4096 * 4
    with pytest.raises(ValueError):
        api.make_config(synth.SHAPES["tiny"], "int8")
    with pytest.raises(ValueError):
        api.make_config(shape, "int4")
    w = api.ModelWeights(1, 1, 1, (api.LayerWeights * 2)(*[api.LayerWeights(1, 1, 1, 1, 1, 1)] * 2))
    h = C.c_void_p()

    def make(**kw):
        d = dict(n_layers=2, hidden=1024, n_heads=8, n_kv_heads=2, head_dim=128, ffn=1024, vocab=1000, rope_theta=1e4,
                 rms_eps=1e-5, dtype=api.SB_INT8)
        d.update(kw)
        return api.lib.sb_model_create(C.byref(api.ModelConfig(*d.values())), C.byref(w), C.byref(h))
    assert make(head_dim=96) == 6 and make(ffn=40000) == 6 and make(n_heads=512) == 6 and make(hidden=1020) == 6
    assert make(dtype=3) == 1
    assert make() == 0
    try:
        sizes = [api.lib.sb_workspace_bytes(h, n, 500) for n in range(1, 257)]
        assert sizes == sorted(sizes) and sizes[0] > 0
        assert api.lib.sb_quantized_workspace_bytes(h, 33, 10, 63) > 0
        assert api.lib.sb_model_set_tap(h, 16, 2, 4) == 0 and api.lib.sb_model_set_tap(h, None, 0, 0) == 0
        par = (C.c_int32 * 1)(-1)
        kv = api.KVCache(16, 16, 64)
        assert api.lib.sb_model_set_forward(h, api.SB_FWD_PERSISTENT) == 0
        assert api.lib.sb_verify_forward(h, C.byref(kv), 4, 16, par, 1, 1.0, 16, 16, 16, 1 << 40, None) == 6
    finally:
        api.lib.sb_model_destroy(h)


def test_binding_refuses_other_types(api):
    with pytest.raises(ValueError, match="rows"):
        api.sb_linear_quantized(torch.zeros(1), torch.zeros((2, 8)), torch.zeros((3, 8)), torch.zeros(1))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        api.sb_linear_quantized(torch.zeros(1), torch.zeros((2, 8), dtype=torch.float16), torch.zeros((2, 8)),
                                torch.zeros(1))
