"""GPU parity of the 8-bit prefix cache with the float64 oracle.

Codes, scales and what a commit moves are exact.  The attention's output is
bfloat16: half a step, 2^-8 of the value; its products see the softmax weights
over 8-bit blocks as binary16, 2^-11 of each weight, so 2^-11 sum p |v| in all.
Scores are float32 sums of head_dim products of 8- by 11-bit numbers: with
|s| <= 64 their error moves a weight by less than head_dim 2^-24 64 = 2^-11
relative in the worst case of every rounding alike.  Together: 2^-8 |o| + 2^-10
sum p |v|, the sums' own float32 roundings far below that.  A weight is held as
p 2^15 vscale / (the largest vscale), and binary16 ends in steps of 2^-24: half
of one is 2^-40 of the largest vscale, times a code of at most its amax, so every
key may be off by 2^-40 of the largest |v| as well (against a largest weight of
1): 2^-40 keys max |v|, seen where a row's weight sits on one key with v = 0.
"""
import numpy as np
import pytest
import torch

from gpu_util import row_relerr, say
from oracle import decoder, quantized, rollback, tree
from paper_2506_01979_amd import synth

pytestmark = pytest.mark.gpu

FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    assert torch.cuda.is_available()
    return A


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16()


def dev(x):
    return x.cuda().contiguous()


def host(x):
    return x.double().cpu().numpy()


def paths(parents):
    on = np.eye(len(parents), dtype=bool)
    for i in range(1, len(parents)):
        on[i] |= on[parents[i]]
    return on


def random_tree(g, n):
    return [-1] + [int(g.integers(max(0, i - 6), i)) for i in range(1, n)]


# ---- blocks ------------------------------------------------------------------------

def special_blocks(g, L, H, slots, d):
    x = g.standard_normal((L, H, slots, d)) * np.exp(g.standard_normal((L, H, 1, d)))
    x = bf16(x).float().numpy()
    x[0, 0, :64] = 0.0                                   # an empty block
    x[0, 1, :64] *= 1e-30                                # tiny, and huge
    x[1, 0, :64] *= 1e30
    x[1, 1, 5, 3] = np.nan
    x[1, 1, 64 + 7, d - 1] = -np.inf
    # ties of int8: amax 254 2^-3, so x 127 / amax = x 4 hits odd halves
    x[0, 0, 64:128] = bf16(g.integers(-254, 255, (64, d)) / 8.0).float().numpy()
    x[0, 0, 64, 0] = 254.0 / 8.0
    return bf16(x)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_quantize_and_back(api, form, d):
    L, H, slots, cap8 = 2, 3, 64 * 5 + 24, 64 * 7
    g = np.random.default_rng(d)
    k, v = special_blocks(g, L, H, slots, d), special_blocks(g, L, H, slots, d)
    cfg = api.attention_config(L, 2 * H, H, d)
    kd, vd = dev(k), dev(v.transpose(2, 3))
    for src_slot, block, n in ((0, 0, 5), (24, 2, 5), (8, 6, 1), (0, 3, 0)):
        say("quantize", form, d, src_slot, block, n)
        c = api.QuantizedKV(cfg, cap8, 64, form)
        for t in (c.k, c.v):
            t.fill_(0x5a)
        for t in (c.k_scale, c.v_scale):
            t.fill_(-5.0)
        api.sb_kv_quantize(cfg, kd, vd, src_slot, c, block, n)
        ko = torch.full((L, H, cap8, d), 7.0, dtype=torch.bfloat16, device="cuda")
        vo = torch.full((L, H, d, cap8), 7.0, dtype=torch.bfloat16, device="cuda")
        api.sb_kv_dequantize(cfg, c, block, n, ko, vo, 64 * block)
        torch.cuda.synchronize()
        inside = slice(64 * block, 64 * (block + n))
        for x, scale, out, raw in ((k, c.k_scale, ko, c.k), (v, c.v_scale, vo.transpose(2, 3), c.v)):
            codes, s = quantized.quantize(x[:, :, src_slot:src_slot + 64 * n].double().numpy(), form)
            got = scale.cpu().numpy()
            assert np.array_equal(got[:, :, block:block + n], s, equal_nan=True)
            assert np.all(got[:, :, :block] == -5.0) and np.all(got[:, :, block + n:] == -5.0)
            assert torch.all(raw[:, :, :block] == 0x5a) and torch.all(raw[:, :, block + n:] == 0x5a)
            ref = bf16(codes.astype(np.float32) * s[..., None, None])       # one float32 product, one rounding
            ref = ref.float().numpy().reshape(L, H, 64 * n, d)
            o = out.float().cpu().numpy()
            assert np.array_equal(o[:, :, inside], ref, equal_nan=True)
            rest = np.ones(cap8, bool)
            rest[inside] = False
            assert np.all(o[:, :, rest] == 7.0)


@pytest.mark.parametrize("tail_len", [0, 1, 63, 64, 65, 100, 128, 191])
@pytest.mark.parametrize("d", [64, 128])
def test_commit(api, d, tail_len):
    L, H, nb0, form = 2, 2, 2, "int8" if tail_len % 2 else "e4m3"
    g = np.random.default_rng(tail_len)
    cfg = api.attention_config(L, H, H, d)
    c = api.QuantizedKV(cfg, 64 * 6, 200, form)
    old = bf16(g.standard_normal((2, L, H, 64 * nb0, d)))
    tail = bf16(g.standard_normal((2, L, H, 200, d)))
    api.sb_kv_quantize(cfg, dev(old[0]), dev(old[1].transpose(2, 3)), 0, c, 0, nb0)
    c.tail_k.copy_(tail[0])
    c.tail_v.copy_(tail[1].transpose(2, 3))
    say("commit", d, tail_len)
    assert api.sb_kv_commit(cfg, c, nb0, tail_len) == (nb0 + tail_len // 64, tail_len % 64)
    n = nb0 + tail_len // 64
    ko = torch.zeros((L, H, 64 * n, d), dtype=torch.bfloat16, device="cuda")
    vo = torch.zeros((L, H, d, 64 * n), dtype=torch.bfloat16, device="cuda")
    api.sb_kv_dequantize(cfg, c, 0, n, ko, vo, 0)
    torch.cuda.synchronize()
    for i, (out, t) in enumerate(((ko, c.tail_k), (vo.transpose(2, 3), c.tail_v.transpose(2, 3)))):
        co, s = quantized.quantize(old[i].double().numpy(), form)
        co, s, left, rest = quantized.commit(co, s, tail[i].double().numpy(), tail_len, form)
        assert rest == tail_len % 64
        ref = bf16(co.astype(np.float32) * s[..., None, None]).double().numpy().reshape(L, H, 64 * n, d)
        assert np.array_equal(host(out), ref)
        assert np.array_equal(host(t), left)              # the slots behind the rest stay as they were


# ---- attention ---------------------------------------------------------------------

def attention_case(api, g, nh, nkv, d, nb, tail, parents, form, layers=1, layer=0, cap_blocks=None, spread=1.0):
    n = len(parents)
    cfg = api.attention_config(layers, nh, nkv, d)
    c = api.QuantizedKV(cfg, 64 * (cap_blocks or nb + 2), tail + n + 16, form)
    c.k_scale.fill_(float("nan"))                          # blocks that no call wrote
    c.v_scale.fill_(float("nan"))
    c.tail_k.fill_(float("nan"))
    c.tail_v.fill_(float("nan"))
    chan = np.exp(0.5 * g.standard_normal((nkv, 1, d)))
    k = bf16(g.standard_normal((nkv, 64 * nb + tail + n, d)) * chan * spread)
    v = bf16(g.standard_normal((nkv, 64 * nb + tail + n, d)) * np.exp(g.standard_normal((nkv, 64 * nb + tail + n, 1))))
    q = bf16(g.standard_normal((n, nh, d)) * np.exp(g.standard_normal((n, nh, 1))))
    ref_k, ref_v = [], []
    for x, ref in ((k, ref_k), (v, ref_v)):
        old = x[:, :64 * nb].double().numpy()
        ref.append(np.concatenate([quantized.values(*quantized.quantize(old, form)) if nb else old,
                                   x[:, 64 * nb:].double().numpy()], 1))
    if nb:
        kk = torch.zeros((layers, nkv, 64 * nb, d), dtype=torch.bfloat16)
        vv = torch.zeros_like(kk)
        kk[layer], vv[layer] = k[:, :64 * nb], v[:, :64 * nb]
        api.sb_kv_quantize(cfg, dev(kk), dev(vv.transpose(2, 3)), 0, c, 0, nb)
    c.tail_k[layer, :, :tail + n] = dev(k[:, 64 * nb:])
    c.tail_v[layer, :, :, :tail + n] = dev(v[:, 64 * nb:].transpose(1, 2))
    ws = torch.full((api.sb_attend_workspace_bytes(cfg, n, nb, tail),), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((n, nh, d), 9.0, dtype=torch.bfloat16, device="cuda")
    return cfg, c, dev(q), out, ws, reference(q, ref_k[0], ref_v[0], parents)


def reference(q, k, v, parents):
    """The output, and how far from it a kernel's may be."""
    out, size = quantized.attend(q.double().numpy(), k, v, paths(parents))
    return out, 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * size + 2.0 ** -40 * v.shape[1] * np.abs(v).max()


def check(out, ref, bound):
    err = np.abs(host(out) - ref)
    assert np.isfinite(err).all()
    at = np.unravel_index(np.argmax(err / bound), err.shape)
    assert err[at] <= bound[at], (at, err[at], bound[at], ref[at])


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("nh,nkv,d", [(4, 4, 64), (8, 2, 64), (4, 4, 128), (16, 2, 128), (6, 1, 128)])
@pytest.mark.parametrize("nb,tail,n", [
    (0, 0, 1), (0, 5, 3), (1, 0, 1), (1, 63, 2), (3, 1, 16), (4, 31, 17), (5, 32, 33), (9, 40, 48),
    (33, 63, 49), (2, 100, 65), (70, 7, 7), (7, 300, 130)])
def test_attend(api, form, nh, nkv, d, nb, tail, n):
    g = np.random.default_rng(1000 * nb + 10 * tail + n)
    parents = random_tree(g, n)
    say("attend", form, nh, nkv, d, nb, tail, n)
    cfg, c, q, out, ws, (ref, bound) = attention_case(api, g, nh, nkv, d, nb, tail, parents, form)
    api.sb_attend_quantized(cfg, c, 0, nb, tail, q, parents, out, ws)
    torch.cuda.synchronize()
    check(out, ref, bound)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("nh,nkv,d,nb,tail,n,layers", [(2, 2, 128, 600, 63, 256, 1), (32, 32, 128, 31, 63, 33, 2),
                                                       (64, 8, 128, 63, 63, 33, 1), (12, 12, 64, 4, 37, 1, 3)])
def test_attend_wide(api, form, nh, nkv, d, nb, tail, n, layers):
    """Whole-chip launches, the largest tree (a chain), a layer other than the first."""
    g = np.random.default_rng(nb)
    parents = list(range(-1, n - 1)) if n == 256 else synth.fork_parents(0, 4, 8) if n == 33 else random_tree(g, n)
    say("attend", form, nh, nkv, d, nb, tail, n)
    cfg, c, q, out, ws, (ref, bound) = attention_case(api, g, nh, nkv, d, nb, tail, parents, form, layers, layers - 1, nb)
    api.sb_attend_quantized(cfg, c, layers - 1, nb, tail, q, parents, out, ws)
    torch.cuda.synchronize()
    check(out, ref, bound)


@pytest.mark.parametrize("form", FORMATS)
def test_attend_extremes(api, form):
    """Zero blocks of K and of V, blocks of very different scales, queries far
    from 1 in size, rows of zeros."""
    g = np.random.default_rng(5)
    nb, tail, n, nkv, d = 12, 3, 20, 2, 128
    parents = random_tree(g, n)
    cfg = api.attention_config(1, 4, nkv, d)
    k = g.standard_normal((nkv, 64 * nb + tail + n, d))
    v = g.standard_normal((nkv, 64 * nb + tail + n, d))
    k[0, 64:128] = 0
    v[:, 128:192] = 0
    v[0, 192:256] *= 1e-12
    v[1, 256:320] *= 1e6
    v[0, :, 5] = 0
    q = g.standard_normal((n, 4, d))
    q[3] = 0
    q[4] *= 1e-12
    q[5, :, ::2] *= 1e-9
    q[6] *= 8
    k, v, q = bf16(k), bf16(v), bf16(q)
    c = api.QuantizedKV(cfg, 64 * nb, tail + n, form)
    cut = 64 * nb
    api.sb_kv_quantize(cfg, dev(k[None, :, :cut]), dev(v[None, :, :cut].transpose(2, 3)), 0, c, 0, nb)
    c.tail_k[0, :, :tail + n] = dev(k[:, cut:])
    c.tail_v[0, :, :, :tail + n] = dev(v[:, cut:].transpose(1, 2))
    ws = torch.empty(api.sb_attend_workspace_bytes(cfg, n, nb, tail), dtype=torch.uint8, device="cuda")
    out = torch.empty((n, 4, d), dtype=torch.bfloat16, device="cuda")
    api.sb_attend_quantized(cfg, c, 0, nb, tail, dev(q), parents, out, ws)
    torch.cuda.synchronize()
    full = [np.concatenate([quantized.values(*quantized.quantize(x[:, :cut].double().numpy(), form)),
                            x[:, cut:].double().numpy()], 1) for x in (k, v)]
    check(out, *reference(q, *full, parents))


def test_attend_shows_a_bad_block(api):
    """A NaN in one KV head's block reaches every row of that head and no other."""
    g = np.random.default_rng(6)
    cfg, c, q, out, ws, (ref, bound) = attention_case(api, g, 4, 2, 64, 3, 2, [-1, 0, 0], "int8")
    c.v_scale[0, 1, 1] = float("nan")
    api.sb_attend_quantized(cfg, c, 0, 3, 2, q, [-1, 0, 0], out, ws)
    torch.cuda.synchronize()
    assert torch.isnan(out[:, 2:]).all() and torch.isfinite(out[:, :2]).all()
    c.v_scale[0, 1, 1] = 0.01
    c.k_scale[0, 0, 2] = float("nan")
    api.sb_attend_quantized(cfg, c, 0, 3, 2, q, [-1, 0, 0], out, ws)
    torch.cuda.synchronize()
    assert torch.isnan(out[:, :2]).all() and torch.isfinite(out[:, 2:]).all()


def test_attend_past_32_bit_offsets(api):
    """The last layer of a cache whose codes take 5.4 GB for K and for V."""
    layers, nkv, nh, d, nb, n, tail = 40, 8, 8, 128, 2048, 3, 4
    parents = [-1, 0, 0]
    cfg = api.attention_config(layers, nh, nkv, d)
    c = api.QuantizedKV(cfg, 64 * nb, 64, "int8")
    assert c.k.numel() > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(3)
    say("attend past 4 GB of codes")
    one = api.attention_config(1, nh, nkv, d)
    k = torch.empty((1, nkv, 64 * nb, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    v = torch.empty((1, nkv, d, 64 * nb), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    small = api.QuantizedKV(one, 64 * nb, 64, "int8")
    api.sb_kv_quantize(one, k, v, 0, small, 0, nb)
    for a, b in ((c.k, small.k), (c.v, small.v), (c.k_scale, small.k_scale), (c.v_scale, small.v_scale)):
        a[layers - 1] = b[0]
    q = torch.empty((n, nh, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    outs = []
    for cf, cache, layer in ((one, small, 0), (cfg, c, layers - 1)):
        cache.tail_k[layer] = 0.25
        cache.tail_v[layer] = -0.5
        out = torch.zeros_like(q)
        ws = torch.empty(api.sb_attend_workspace_bytes(cf, n, nb, tail), dtype=torch.uint8, device="cuda")
        api.sb_attend_quantized(cf, cache, layer, nb, tail, q, parents, out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    ko = torch.zeros_like(k)
    vo = torch.zeros_like(v)
    api.sb_kv_dequantize(one, small, 0, nb, ko, vo, 0)
    kk, vv = ko[0, 3].double(), vo[0, 3].t().double()
    s = torch.cat([q[1:2, 3].double() @ kk.t(), (q[1:2, 3].double().sum(-1, keepdim=True) * 0.25).expand(1, tail + 2)], 1)
    p = torch.softmax(s / d ** 0.5, -1)
    ref = p[:, :64 * nb] @ vv - 0.5 * p[:, 64 * nb:].sum()
    size = p[:, :64 * nb] @ vv.abs() + 0.5 * p[:, 64 * nb:].sum()
    # the dequantised values carry a bfloat16 rounding of their own: K's moves a
    # score by up to 2^-8 sum |q k| / sqrt d and V's an entry by 2^-8
    err = (outs[1][1, 3].double() - ref[0]).abs()
    assert bool((err <= 2 ** -8 * ref[0].abs() + 2 ** -5 * size[0]).all())
    del c, small
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", FORMATS)
def test_attend_captured_and_on_a_stream(api, form):
    """Replays of a captured call follow the buffers' contents, with eager work between."""
    g = np.random.default_rng(8)
    parents = random_tree(g, 40)
    cfg, c, q, out, ws, (ref, bound) = attention_case(api, g, 4, 2, 128, 6, 20, parents, form)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        api.sb_attend_quantized(cfg, c, 0, 6, 20, q, parents, out, ws)
    q2 = q.clone()
    other, ws2 = torch.empty_like(out), torch.empty_like(ws)
    for i in range(4):
        q.copy_(q2 * (1.0 if i % 2 else 0.5))
        out.zero_()
        graph.replay()
        api.sb_attend_quantized(cfg, c, 0, 6, 20, q, parents, other, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, other)
    check(out, ref, bound)
    with torch.cuda.stream(st):
        out.zero_()
        api.sb_attend_quantized(cfg, c, 0, 6, 20, q, parents, out, ws)
    st.synchronize()
    assert torch.equal(out, other)
    out.zero_()
    torch.cuda.synchronize()
    api.sb_attend_quantized(cfg, c, 0, 6, 20, q, parents, out, ws, stream=st)
    st.synchronize()
    assert torch.equal(out, other)


# ---- the forward on it ------------------------------------------------------------------

@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("sname,nb,tail,parents", [
    ("small_bf16", 2, 9, [-1, 0, 0, 1, 2]), ("small_gqa_bf16", 1, 63, synth.fork_parents(2, 3, 4)),
    ("small_h128_bf16", 3, 0, synth.fork_parents(0, 4, 8)), ("ragged_bf16", 2, 30, [-1]),
    ("gqa128_bf16", 0, 12, [-1, 0, 1, 1]), ("small_gqa128_bf16", 2, 17, list(range(-1, 70)))])
def test_forward(api, form, sname, nb, tail, parents):
    """The verify forward against the oracle decoder on the values that the cache
    stands for: logits to 2e-2 of the row's largest and the tail rows' K/V alike,
    the bound of a bfloat16 forward in this framework's tests."""
    shape = synth.SHAPES[sname]
    W = synth.model_weights(shape)
    m = api.Model(shape, api.dict_tensors(W))
    n, P = len(parents), 64 * nb + tail
    g = np.random.default_rng(P)
    Kp = bf16(g.standard_normal((shape.n_layers, shape.n_kv_heads, P, shape.head_dim))).float().numpy()
    Vp = bf16(g.standard_normal(Kp.shape)).float().numpy()
    tokens = g.integers(0, shape.vocab, n).astype(np.int32)
    c = api.QuantizedKV(m.cfg, 64 * nb + 64, tail + n + 8, form)
    c.tail_k.fill_(float("nan"))
    c.tail_v.fill_(float("nan"))
    k, v = m.new_kv(max(P, 8))
    if P:
        m.load_kv(k, v, Kp, Vp, P)
    api.sb_kv_quantize(m.cfg, k, v, 0, c, 0, nb)
    c.tail_k[:, :, :tail] = k[:, :, 64 * nb:P]
    c.tail_v[:, :, :, :tail] = v[:, :, :, 64 * nb:P]
    logits = torch.empty((n, shape.vocab), dtype=torch.float32, device="cuda")
    stats = api.new_stats(n)
    ws = m.quantized_workspace(n, nb, tail)
    say("forward", form, sname, nb, tail, n)
    m.sb_verify_forward_quantized(c, nb, tail, torch.from_numpy(tokens).cuda(), parents, 1.0, logits, stats, ws)
    torch.cuda.synchronize()
    seen = [np.concatenate([quantized.values(*quantized.quantize(x[:, :, :64 * nb], form)) if nb else x[:, :, :0],
                            x[:, :, 64 * nb:]], 2).astype(np.float32) for x in (Kp, Vp)]
    ref, kt, vt = decoder.tree_forward(shape, W, *seen, P, tokens, parents, "bf16")
    assert row_relerr(logits.cpu().numpy(), ref) < 2e-2
    K2, V2 = m.read_kv(c.tail_k, c.tail_v, tail, n)
    assert row_relerr(K2.reshape(-1, shape.head_dim), kt.reshape(-1, shape.head_dim)) < 2e-2
    assert row_relerr(V2.reshape(-1, shape.head_dim), vt.reshape(-1, shape.head_dim)) < 2e-2
    st = api.decode_stats(stats)
    assert np.array_equal(st["argmax"], logits.cpu().numpy().argmax(-1))


def test_forward_without_blocks_is_the_forward(api):
    """With every token in the tail, the two forwards see the same cache."""
    shape = synth.SHAPES["small_h128_bf16"]
    m = api.Model(shape, api.synth_tensors(shape))
    parents, P = synth.fork_parents(1, 3, 5), 50
    n = len(parents)
    g = torch.Generator(device="cuda").manual_seed(2)
    c = api.QuantizedKV(m.cfg, 64, P + n, "int8")
    c.tail_k.normal_(generator=g)
    c.tail_v.normal_(generator=g)
    k, v = c.tail_k.clone(), c.tail_v.clone()
    toks = torch.randint(0, shape.vocab, (n,), dtype=torch.int32, device="cuda", generator=g)
    a, b = (torch.empty((n, shape.vocab), dtype=torch.float32, device="cuda") for _ in range(2))
    m.sb_verify_forward(k, v, P, toks, parents, 1.0, a, api.new_stats(n), m.workspace(n, P))
    m.sb_verify_forward_quantized(c, 0, P, toks, parents, 1.0, b, api.new_stats(n), m.quantized_workspace(n, 0, P))
    torch.cuda.synchronize()
    # the same attention in another order of sums: within the framework's own
    # bound for that (bfloat16 roundings that fall the other way)
    assert row_relerr(b.cpu().numpy(), a.cpu().numpy()) < 2e-2
    assert row_relerr(c.tail_k.float().cpu().numpy().reshape(-1, 128), k.float().cpu().numpy().reshape(-1, 128)) < 2e-2


def test_steps_together(api):
    """Verify, walk, rollback and commit, step after step from an empty cache:
    the lengths, the tail and the blocks follow the oracle's, which keeps every
    committed token's K/V as the GPU wrote it."""
    shape, form = synth.SHAPES["small_gqa_bf16"], "e4m3"
    m = api.Model(shape, api.synth_tensors(shape))
    L, H, d, V = shape.n_layers, shape.n_kv_heads, shape.head_dim, shape.vocab
    parents = synth.fork_parents(20, 2, 3)
    n = len(parents)
    cap = 64 + n
    c = api.QuantizedKV(m.cfg, 256, cap, form)
    cap = c.tail_k.shape[2]
    ws = m.quantized_workspace(n, 4, 63)
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.empty((n, V), dtype=torch.float32, device="cuda")
    stats, res, new_len = api.new_stats(n), api.new_result(), torch.zeros(1, dtype=torch.int32, device="cuda")
    sws = torch.empty(api.sb_sample_workspace_bytes(V), dtype=torch.uint8, device="cuda")
    tokens = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda", generator=g)
    nb = tail = total = 0
    codes = [np.zeros((L, H, 0, 64, d)) for _ in range(2)]
    scales = [np.zeros((L, H, 0), np.float32) for _ in range(2)]
    for step in range(14):
        m.sb_verify_forward_quantized(c, nb, tail, tokens, parents, 1.0, logits, stats, ws)
        # drafts that are accepted often: q is p but for its scale
        q = torch.softmax(logits, -1)[np.maximum(parents, 0)]
        u = torch.rand(n, device="cuda", generator=g) * (0.4 if step % 3 else 1.0)
        api.sb_accept_resample(tokens, parents, logits, stats, 1.0, q, u, res, sws)
        torch.cuda.synchronize()
        path = api.decode_result(res)["path"]
        before = [host(c.tail_k), host(c.tail_v.transpose(2, 3))]
        m.sb_kv_rollback(c.tail_k, c.tail_v, tail, res, new_len)
        tail2 = int(new_len.item())
        assert tail2 == tail + len(path)
        total += len(path)
        say("step", step, "accepted", len(path) - 1, "cache", 64 * nb + tail2)
        want = rollback.kv_rollback(*before, tail, path)[:2]
        nb, rest = api.sb_kv_commit(m.cfg, c, nb, tail2)
        for i in range(2):
            codes[i], scales[i], want_tail, tl = quantized.commit(codes[i], scales[i], want[i], tail2, form)
            assert tl == rest and codes[i].shape[2] == nb
            got = host(c.tail_k if i == 0 else c.tail_v.transpose(2, 3))
            assert np.array_equal(got[:, :, :rest], want_tail[:, :, :rest])
        tail = rest
        assert 64 * nb + tail == total
        if nb == 3:
            break
        tokens = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda", generator=g)
        tokens[0] = api.decode_result(res)["next_token"]
    assert nb >= 1
    ko = torch.zeros((L, H, 64 * nb, d), dtype=torch.bfloat16, device="cuda")
    vo = torch.zeros((L, H, d, 64 * nb), dtype=torch.bfloat16, device="cuda")
    api.sb_kv_dequantize(m.cfg, c, 0, nb, ko, vo, 0)
    torch.cuda.synchronize()
    for i, out in enumerate((ko, vo.transpose(2, 3))):
        ref = bf16(codes[i].astype(np.float32) * scales[i][..., None, None]).double().numpy().reshape(L, H, -1, d)
        assert np.array_equal(host(out), ref)
    assert tree.depths(np.asarray(parents)).max() == 23
