"""GPU tests of the 8-bit cache where it can go wrong: the largest finite values,
the bits of the softmax weights, values that are not finite, and forms of the
attention that only long prefixes take."""
import numpy as np
import pytest
import torch

from attend_forms import MANY_BLOCKS, THREE_TILES, plan
from gpu_util import say
from oracle import quantized
from paper_2506_01979_amd import synth
from test_gpu_quantized import bf16, check, dev, host, random_tree, reference

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


# ---- attention ---------------------------------------------------------------------

def exact_cache(api, g, form, nh, nkv, d, nb, tail, parents, layers=1):
    """A cache whose values the 8-bit type holds exactly (codes times powers of two),
    queries of small whole numbers: scores and their sums are exact in float32."""
    n, keys = len(parents), 64 * nb + tail + len(parents)
    top = quantized.TOP[form]

    def values(step):
        x = quantized.nearest(g.uniform(-top / 2, top / 2, (nkv, keys, d)), form)
        x[:, 5:64 * nb:64, 0] = top                        # every block's largest
        return bf16(x * step)
    k, v = values(2.0 ** -3), values(2.0 ** -9)
    q = bf16(g.integers(-2, 3, (n, nh, d)) * (1.0 if form == "int8" else 0.25))
    cfg = api.attention_config(layers, nh, nkv, d)
    c = api.QuantizedKV(cfg, 64 * max(nb, 1), tail + n, form)
    cut = 64 * nb
    if nb:
        api.sb_kv_quantize(cfg, dev(k[None, :, :cut]), dev(v[None, :, :cut].transpose(2, 3)), 0, c, 0, nb)
        for x in (k, v):
            codes, s = quantized.quantize(x[:, :cut].double().numpy(), form)
            assert np.array_equal(quantized.values(codes, s), x[:, :cut].double().numpy())
    c.tail_k[0, :, :tail + n] = dev(k[:, cut:])
    c.tail_v[0, :, :, :tail + n] = dev(v[:, cut:].transpose(1, 2))
    return cfg, c, k, v, q


def attend(api, cfg, c, nb, tail, q, parents):
    n = len(parents)
    ws = torch.full((api.sb_attend_workspace_bytes(cfg, n, nb, tail),), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    api.sb_attend_quantized(cfg, c, 0, nb, tail, dev(q), parents, out, ws)
    torch.cuda.synchronize()
    return out


def on_path(parents):
    on = np.eye(len(parents), dtype=bool)
    for i in range(1, len(parents)):
        on[i] |= on[parents[i]]
    return on


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("nh,nkv,d,nb,tail,n", [(4, 4, 64, 3, 1, 1), (8, 2, 64, 9, 40, 17), (8, 2, 128, 1, 0, 1),
                                                (4, 2, 128, 20, 33, 33), (2, 2, 128, 130, 5, 129), (2, 1, 64, 130, 5, 88)])
def test_attend_keeps_the_weights(api, form, nh, nkv, d, nb, tail, n):
    """The output is the bfloat16 nearest to a value that is within 2^-15 sum p |v| of the
    exact one.  What the scores and weights lose on the way: K, V and q enter exactly
    and the sums of q k are exact, as every term is a multiple of one step and they
    stay below 2^24 of them.  A score in the softmax's units of log 2 is below 64 in
    size; its factor is three roundings (3 2^-24), the sum with the maximum one more
    of a number below 128 (2^-18), both times log 2: 2^-17.4 of a weight at most.  The
    exponential, 1 / r and log r: 2^-20.  A weight in two parts of 8 or of 11 bits keeps
    2^-18.  Sums of at most 2^14 weights in float32, in four or more parts: 2^-24 times
    their steps, 2^-17 if they all fall one way.  Together below 2^-15.  (Weights of 11
    bits: 2^-12 on the average of a weight.)"""
    g = np.random.default_rng(100 * nb + n)
    parents = random_tree(g, n)
    say("attend, weights", form, nh, nkv, d, nb, tail, n)
    cfg, c, k, v, q = exact_cache(api, g, form, nh, nkv, d, nb, tail, parents)
    out = host(attend(api, cfg, c, nb, tail, q, parents))
    ref, size = quantized.attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), on_path(parents))
    delta = 2.0 ** -15 * size
    low, high = (nearest_bf16(ref + f * delta) for f in (-1, 1))
    assert ((out >= low) & (out <= high)).all(), (np.mean((out < low) | (out > high)), np.abs((out - ref) / size).max())


def nearest_bf16(x):
    """float64 to the nearest bfloat16 in one rounding, ties to even."""
    _, e = np.frexp(x)
    step = np.ldexp(1.0, e - 8)
    return np.rint(x / step) * step


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("nh,nkv,d,nb,tail,n,bad", [(4, 2, 64, 6, 9, 5, 3), (4, 2, 128, 12, 40, 33, 39), (128, 64, 64, 130, 9, 5, 3),
                                                    (64, 64, 128, 130, 70, 20, 0)])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_attend_value_not_finite_in_the_tail(api, form, nh, nkv, d, nb, tail, n, bad, value):
    """One value of a committed tail slot that is not finite: every row attends to
    it and shows it in that dimension, the others are what they are without it (with
    many heads a wave goes on from the tail to blocks)."""
    g = np.random.default_rng(nb + n)
    parents = random_tree(g, n)
    cfg, c, k, v, q = exact_cache(api, g, form, nh, nkv, d, nb, tail, parents)
    say("attend, not finite in the tail", form, nh, nkv, d, nb, tail, n, bad, value)
    without = attend(api, cfg, c, nb, tail, q, parents)
    c.tail_v[0, 1, 17, bad] = value
    out = attend(api, cfg, c, nb, tail, q, parents)
    hit = slice(nh // nkv, 2 * (nh // nkv))
    shown = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    shown[:, hit, 17] = True
    assert not torch.isfinite(out[shown]).any()
    # the sums of a wave may be kept in another unit: float32 roundings, then one bfloat16 step
    a, b = host(out[~shown]), host(without[~shown])
    assert np.isfinite(a).all() and (np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 1e-5).all()


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("d,nb,tail,n", [(64, 6, 9, 20), (128, 12, 40, 33), (128, 130, 62, 129), (64, 0, 0, 12)])
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_attend_row_not_finite_off_the_path(api, form, d, nb, tail, n, value):
    """A tree row whose K and V are not finite: the rows on whose path it stands show
    it, the others are what they are without it."""
    g = np.random.default_rng(nb + n)
    parents = random_tree(g, n)
    cfg, c, k, v, q = exact_cache(api, g, form, 4, 2, d, nb, tail, parents)
    say("attend, not finite beside the path", form, d, nb, tail, n, value)
    without = attend(api, cfg, c, nb, tail, q, parents)
    bad = n // 2
    c.tail_k[0, 0, tail + bad, 5] = value
    c.tail_v[0, 0, 11, tail + bad] = value
    c.tail_v[0, 1, :, tail + bad] = value
    out = attend(api, cfg, c, nb, tail, q, parents)
    sees = torch.from_numpy(on_path(parents)[:, bad].copy()).cuda()
    assert 1 <= int(sees.sum()) < n
    a, b = host(out[~sees]), host(without[~sees])
    assert np.isfinite(a).all() and (np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 1e-5).all()
    assert not torch.isfinite(out[sees][:, 2:]).any() and not torch.isfinite(out[sees][:, :2, 11]).any()


@pytest.mark.parametrize("projections", [None, "int8"])
def test_forward_with_a_row_not_finite(api, projections):
    """A draft token whose embedding is not finite: its row and its descendants show it,
    the others' logits, statistics and tail K/V are what they are without it."""
    shape = synth.SHAPES["small_gqa_bf16"]
    parents, nb, tail = synth.fork_parents(1, 3, 4), 2, 11
    n, V = len(parents), shape.vocab
    m = api.Model(shape, api.synth_tensors(shape), projections=projections)
    g = torch.Generator(device="cuda").manual_seed(7)
    c = api.QuantizedKV(m.cfg, 64 * nb, tail + n, "int8")
    k, v = m.new_kv(64 * nb)
    k.normal_(generator=g)
    v.normal_(generator=g)
    api.sb_kv_quantize(m.cfg, k, v, 0, c, 0, nb)
    c.tail_k.normal_(generator=g)
    c.tail_v.normal_(generator=g)
    tokens = torch.arange(n, dtype=torch.int32, device="cuda")
    ws = m.quantized_workspace(n, nb, tail)
    bad, outs = 3, []
    for value in (None, float("nan")):
        if value is not None:
            m.embed[bad, 5] = value
        logits, stats = torch.empty((n, V), device="cuda"), api.new_stats(n)
        say("forward, a row not finite", projections, value)
        m.sb_verify_forward_quantized(c, nb, tail, tokens, parents, 1.0, logits, stats, ws)
        torch.cuda.synchronize()
        outs.append((logits, stats.clone(), c.tail_k[:, :, tail:tail + n].clone(), c.tail_v[..., tail:tail + n].clone()))
    sees = torch.from_numpy(on_path(parents)[:, bad].copy()).cuda()
    assert 2 <= int(sees.sum()) < n
    (l0, s0, k0, v0), (l1, s1, k1, v1) = outs
    assert torch.equal(l1[~sees], l0[~sees]) and torch.equal(s1[~sees], s0[~sees])
    assert torch.equal(k1[:, :, ~sees], k0[:, :, ~sees]) and torch.equal(v1[..., ~sees], v0[..., ~sees])
    assert torch.isfinite(l0).all() and not torch.isfinite(l1[sees]).any()


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("nh,nkv,d,nb,tail,n", THREE_TILES + MANY_BLOCKS)
def test_attend_long(api, form, nh, nkv, d, nb, tail, n):
    """Blocks of very different scales, a wave's largest V scale in its last ones: the
    oracle's output on the first and the last KV head, to the bound of the other
    attention tests."""
    g = torch.Generator(device="cuda").manual_seed(nb + n)
    parents = random_tree(np.random.default_rng(n), n)
    say("attend, long", form, nh, nkv, d, nb, tail, n, plan(nh, nkv, d, nb, tail, n))
    cfg, cut, keys = api.attention_config(1, nh, nkv, d), 64 * nb, 64 * nb + tail + n
    size = torch.exp(torch.empty((2, 1, nkv, keys // 64 + 1, 1, 1), device="cuda").normal_(generator=g))
    size[1, :, :, nb - 5:nb] *= 32.0
    k, v = ((torch.empty((1, nkv, len(size[0, 0, 0]) * 64, d), device="cuda").normal_(generator=g).view(1, nkv, -1, 64, d)
             * s).view(1, nkv, -1, d)[:, :, :keys].bfloat16() for s in size)
    q = torch.empty((n, nh, d), device="cuda").normal_(generator=g).bfloat16()
    c = api.QuantizedKV(cfg, cut, tail + n, form)
    api.sb_kv_quantize(cfg, k[:, :, :cut].contiguous(), v[:, :, :cut].transpose(2, 3).contiguous(), 0, c, 0, nb)
    c.tail_k[:, :, :tail + n] = k[:, :, cut:]
    c.tail_v[:, :, :, :tail + n] = v[:, :, cut:].transpose(2, 3)
    out = attend(api, cfg, c, nb, tail, q, parents)
    G = nh // nkv
    for h in (0, nkv - 1):
        kk, vv = (np.concatenate([quantized.values(*quantized.quantize(host(x[0, h, :cut]), form)), host(x[0, h, cut:])])
                  for x in (k, v))
        heads = slice(h * G, (h + 1) * G)
        check(out[:, heads], *reference(q[:, heads].cpu(), kk[None], vv[None], parents))
