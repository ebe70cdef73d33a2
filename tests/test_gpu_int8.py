"""GPU parity of the 8-bit projections and of the forward on them.

The product is exact in integers and its scales round in a fixed order, so y is
the oracle's bit for bit.

Over a whole forward the last bits of the float32 values between the products
differ, some codes and bfloat16 values fall the other way, and from there on
every quantisation rounds afresh: two right forwards end as far apart as either is
from the unquantised one (in float64, the oracle with inputs 1e-6 apart: 0.015 to
0.05 of a row's largest logit).  By arithmetic: a Gaussian input of 256 to 1024 values has
amax about 3.2 sigma, a step of 3.2 / 127 sigma and a rounding of that / sqrt 12
= 0.73 %, two roundings apart 1.03 %; the product silu(gate) up has amax about
10 sigma, 3.2 %.  Seven inputs of the first kind and two of the second on
the way to the logits of two layers: sqrt(7 1.03^2 + 2 3.2^2) = 5.3 % of their norm;
the largest of some thousand errors is about 4.5 sigma where the largest logit is
about 3.2: 7.4 %, so 8e-2.  What must also hold, and tells a mistake from
rounding: the kernel's logits are as near to the unquantised forward's as the oracle's
are (1.5 times, for the two draws of one spread), and the first layer's keys and
values, which one quantisation and one bfloat16 rounding separate from the
embedding, agree to a bfloat16 step, 2^-7, and a code here and there, in all 1e-2."""
import numpy as np
import pytest
import torch

from gpu_util import row_relerr, say
from oracle import decoder, int8, quantized
from paper_2506_01979_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    assert torch.cuda.is_available()
    return A


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16()


def product(api, w, x, shift=0):
    """y of one call, in a buffer whose surroundings must stay as they are."""
    (m, k), n = w.shape, len(x)
    packed = torch.full((api.sb_linear_packed_bytes(m, k),), 0x55, dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(w.cuda(), packed)
    buf = torch.full((n * m + 64 + shift,), 7.0, device="cuda")
    y = buf[shift:shift + n * m].view(n, m)
    ws = torch.full((api.sb_linear_workspace_bytes(m, k, n),), 0xff, dtype=torch.uint8, device="cuda")
    api.sb_linear_quantized(packed, x.cuda(), y, ws)
    torch.cuda.synchronize()
    assert (buf[:shift] == 7.0).all() and (buf[shift + n * m:] == 7.0).all()
    return y.cpu().numpy()


def inputs(g, m, k, n, f32):
    w = bf16(g.standard_normal((m, k)) * np.exp(g.standard_normal((m, 1))))
    x = g.standard_normal((n, k)) * np.exp(g.standard_normal((n, 1))) * np.exp(g.standard_normal((1, k)))
    return w, (torch.from_numpy(x.astype(np.float32)) if f32 else bf16(x))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,k", [(1, 1), (5, 8), (16, 63), (17, 64), (100, 65), (1000, 328), (250, 1032), (4096, 512),
                                 (48, 11008), (33, 32768), (9001, 264)])
@pytest.mark.parametrize("n", [1, 3, 16, 17, 33, 64, 65, 81, 129, 200, 256])
def test_linear(api, f32, m, k, n):
    g = np.random.default_rng(m + 3 * k + 7 * n)
    say("linear", m, k, n, f32)
    w, x = inputs(g, m, k, n, f32)
    got = product(api, w, x, shift=n % 3)
    ref = int8.linear(x.float().numpy(), w.float().numpy(), np.float32 if f32 else np.float64)
    assert np.array_equal(got, ref)


@pytest.mark.parametrize("m,k,rows", [
    (22005, 1160, (48, 49, 81, 97, 129, 180, 193, 256)),  # 128 channels a workgroup, whole K
    (5003, 5128, (48, 64, 65, 130, 200, 256)),            # and six K ranges, the last channels' group short
    (40001, 650, (49, 81, 98, 129, 177, 255)),            # 256 channels
    (3001, 8200, (100, 193, 256)),                        # eight K ranges of 128 channels' groups
    (8001, 8200, (193, 256)),                             # and of 256 channels'
    (5120, 13130, (16, 17, 33, 47)),                      # a long K and an uneven split of the channels
    (76810, 500, (50, 256)),                              # more workgroups than one round
    (8200, 32768, (48, 60)),                              # the longest K, offsets of a tile group near 8 MB
])
def test_linear_large(api, m, k, rows):
    """Matrices past 24 MB of codes: the workgroups share stages of both operands, and K ranges
    of one product meet in the workspace.  Exact against the oracle on 400 channels, the first
    and last among them; on a workspace sized for the most rows and full of other bytes."""
    g = torch.Generator().manual_seed(m + k)
    w = torch.randn((m, k), generator=g).bfloat16()
    some = torch.cat([torch.arange(150), torch.randint(150, m - 150, (100,), generator=g), torch.arange(m - 150, m)])
    packed = torch.full((api.sb_linear_packed_bytes(m, k),), 0x55, dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(w.cuda(), packed)
    sizes = [api.sb_linear_workspace_bytes(m, k, n) for n in range(1, 257)]
    assert sizes == sorted(sizes)
    ws = torch.full((sizes[rows[-1] - 1],), 0xff, dtype=torch.uint8, device="cuda")
    wf = w[some].float().numpy()
    for n in rows:
        say("large linear", m, k, n)
        x = torch.randn((n, k), generator=g).bfloat16()
        buf = torch.full((n * m + 64,), 7.0, device="cuda")
        y = buf[:n * m].view(n, m)
        api.sb_linear_quantized(packed, x.cuda(), y, ws)
        assert (buf[n * m:] == 7.0).all()
        assert np.array_equal(y[:, some.cuda()].cpu().numpy(), int8.linear(x.float().numpy(), wf))


@pytest.mark.parametrize("m,k", [(8180, 330), (11000, 260), (17601, 130), (22000, 200), (24400, 520), (30001, 66), (57000, 72)])
@pytest.mark.parametrize("n", [1, 16, 17, 33, 50, 70, 100, 150])
def test_linear_tiles(api, m, k, n):
    """One to eight weight tiles a workgroup: one even round of them, or several."""
    g = torch.Generator().manual_seed(m + k + n)
    say("linear tiles", m, k, n)
    w, x = torch.randn((m, k), generator=g).bfloat16(), torch.randn((n, k), generator=g)
    got = product(api, w, x, shift=4 * (n % 2))
    assert np.array_equal(got, int8.linear(x.numpy(), w.float().numpy(), np.float32))


@pytest.mark.parametrize("m,k", [(1030, 13800), (57500, 1030)])
@pytest.mark.parametrize("n", [17, 33, 50, 70, 100, 140, 190, 256])
def test_linear_shared_stages(api, m, k, n):
    """Every number of token tiles that workgroups share, on K ranges of one product and on whole
    ones of 256 channels a workgroup."""
    g = torch.Generator().manual_seed(m + k + n)
    say("linear shared", m, k, n)
    w, x = torch.randn((m, k), generator=g).bfloat16(), torch.randn((n, k), generator=g).bfloat16()
    got = product(api, w, x, shift=n % 4)
    assert np.array_equal(got, int8.linear(x.float().numpy(), w.float().numpy()))


def test_linear_k_ranges_captured(api):
    """K ranges and their join replayed, beside eager calls on a workspace of their own."""
    m, k, n = 1030, 13800, 70
    assert api.sb_linear_workspace_bytes(m, k, n) > 2 ** 20 + 80 * 13824
    g = torch.Generator().manual_seed(6)
    packed = torch.empty(api.sb_linear_packed_bytes(m, k), dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(torch.randn((m, k), generator=g).bfloat16().cuda(), packed)
    x0 = torch.randn((n, k), generator=g).cuda()
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


def test_linear_large_captured(api):
    """K ranges and their join in a graph, beside eager calls on a workspace of their own."""
    m, k, n = 5003, 5128, 70
    g = torch.Generator().manual_seed(5)
    packed = torch.empty(api.sb_linear_packed_bytes(m, k), dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(torch.randn((m, k), generator=g).bfloat16().cuda(), packed)
    x0 = torch.randn((n, k), generator=g).cuda()
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


def test_linear_special_rows(api):
    """Zero rows and channels, NaN and infinity in one: they stay where they are."""
    g = np.random.default_rng(1)
    w, x = inputs(g, 40, 130, 20, False)
    w[3], x[4], w[5, 7], x[6, 129], x[7, 0] = 0, 0, float("inf"), float("nan"), float("-inf")
    x[9] = x[9] * 1e-37
    w[11] = w[11] * 1e-30
    got = product(api, w, x)
    ref = int8.linear(x.float().numpy(), w.float().numpy())
    assert np.array_equal(got, ref, equal_nan=True)
    assert np.isnan(got[6:8]).all() and np.isnan(got[:, 5]).all() and np.isfinite(got[0, :5]).all()


def test_linear_largest_sums(api):
    """Every code 127: 32768 of them sum to 5.3e8, in 32 bits."""
    w, x = torch.ones((20, 32768), dtype=torch.bfloat16), torch.ones((3, 32768), dtype=torch.bfloat16)
    x[1] = -1
    got = product(api, w, x)
    s = np.float32(1) / np.float32(127)
    assert np.array_equal(got[0], np.full(20, np.float32(127 * 127 * 32768) * (s * s), np.float32))
    assert np.array_equal(got[1], -got[0])


def test_linear_captured_and_on_a_stream(api):
    g = np.random.default_rng(2)
    w, x = inputs(g, 300, 512, 40, False)
    packed = torch.empty(api.sb_linear_packed_bytes(300, 512), dtype=torch.uint8, device="cuda")
    api.sb_linear_pack(w.cuda(), packed)
    x0 = x.cuda()
    xd, y, y2 = x0.clone(), torch.zeros((40, 300), device="cuda"), torch.zeros((40, 300), device="cuda")
    ws, ws2 = (torch.empty(api.sb_linear_workspace_bytes(300, 512, 40), dtype=torch.uint8, device="cuda") for _ in range(2))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        api.sb_linear_quantized(packed, xd, y, ws)
    for i in range(4):
        xd.copy_(x0 * (2.0 if i % 2 else -1.0))
        y.zero_()
        graph.replay()
        api.sb_linear_quantized(packed, xd, y2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(y, y2)
    torch.cuda.synchronize()
    y.zero_()
    torch.cuda.synchronize()
    api.sb_linear_quantized(packed, xd, y, ws, stream=st)
    st.synchronize()
    assert torch.equal(y, y2)


# ---- the model -----------------------------------------------------------------------

_WEIGHTS = {}


def weights(shape):
    if shape.name not in _WEIGHTS:
        _WEIGHTS[shape.name] = synth.model_weights(shape)
    return _WEIGHTS[shape.name]


def gains(W, g):
    """The weights with norm gains other than 1."""
    W = dict(W, layers=[dict(l) for l in W["layers"]])
    for d, names in [(W, ["final_norm"])] + [(l, ["attn_norm", "mlp_norm"]) for l in W["layers"]]:
        for n in names:
            d[n] = (1 + 0.2 * g.standard_normal(d[n].shape)).astype(np.float32)
    return W


def check_logits(got, ref, plain):
    assert row_relerr(got, ref) < 8e-2
    far = [float(np.linalg.norm(x - plain) / np.linalg.norm(plain)) for x in (got, ref)]
    assert far[0] <= 1.5 * far[1] + 1e-6, far


@pytest.mark.parametrize("sname,P,parents", [
    ("small_bf16", 40, [-1]), ("small_bf16", 0, [-1, 0, 0, 1]), ("small_gqa_bf16", 33, synth.fork_parents(2, 3, 4)),
    ("small_h128_bf16", 100, synth.fork_parents(0, 4, 8)), ("ragged_bf16", 21, synth.fork_parents(1, 2, 2)),
    ("small_gqa128_bf16", 70, list(range(-1, 80)))])
def test_forward(api, sname, P, parents):
    shape, n, g = synth.SHAPES[sname], len(parents), np.random.default_rng(P)
    W = gains(weights(shape), g)
    say("int8 forward", sname, P, n)
    m = api.Model(shape, api.dict_tensors(W), projections="int8")
    K = bf16(g.standard_normal((shape.n_layers, shape.n_kv_heads, P, shape.head_dim))).float().numpy()
    V = bf16(g.standard_normal(K.shape)).float().numpy()
    tokens = g.integers(0, shape.vocab, n).astype(np.int32)
    k, v = m.new_kv(P + n + 8)
    k.fill_(float("nan"))
    v.fill_(float("nan"))
    if P:
        m.load_kv(k, v, K, V, P)
    logits, stats = torch.empty((n, shape.vocab), device="cuda"), api.new_stats(n)
    taps = torch.zeros((2, n, shape.hidden), device="cuda")
    m.sb_model_set_tap(taps, 2, n)
    m.sb_verify_forward(k, v, P, torch.from_numpy(tokens).cuda(), parents, 1.0, logits, stats, m.workspace(n, P))
    torch.cuda.synchronize()
    hidden = []
    ref, kt, vt = int8.tree_forward(shape, W, K, V, P, tokens, parents, hidden)
    check_logits(logits.cpu().numpy(), ref, decoder.tree_forward(shape, W, K, V, P, tokens, parents, "bf16")[0])
    flat = lambda x: x.reshape(-1, shape.head_dim)  # noqa: E731
    for got, want in zip(m.read_kv(k, v, P, n), (kt, vt)):
        assert row_relerr(flat(got[0]), flat(want[0])) < 1e-2 and row_relerr(flat(got[1]), flat(want[1])) < 8e-2
    last = hidden[1] * decoder.rms_scale(hidden[1], shape.rms_eps, np.float64) * W["final_norm"]
    assert row_relerr(taps[0].cpu().numpy(), hidden[0]) < 8e-2 and row_relerr(taps[1].cpu().numpy(), last) < 8e-2
    assert np.array_equal(api.decode_stats(stats)["argmax"], logits.cpu().numpy().argmax(-1))


def test_forward_with_k_ranges(api):
    """A long FFN on a narrow hidden size: the down projection takes K ranges, whose sums stand
    in the step's workspace (full of other bytes here), and is followed by the norm."""
    shape = synth.Shape("wide_ffn", 1, 1024, 8, 8, 128, 13824, 1000, "bf16")
    n, P, parents = 33, 20, synth.branch_parents(4, 8)
    assert api.sb_linear_workspace_bytes(1024, 13824, n) > 2 ** 20 + 48 * 13824
    g = np.random.default_rng(41)
    W = gains(weights(shape), g)
    m = api.Model(shape, api.dict_tensors(W), projections="int8")
    K = bf16(g.standard_normal((1, 8, P, 128))).float().numpy()
    V = bf16(g.standard_normal(K.shape)).float().numpy()
    tokens = g.integers(0, shape.vocab, n).astype(np.int32)
    k, v = m.new_kv(P + n)
    m.load_kv(k, v, K, V, P)
    logits, stats = torch.empty((n, shape.vocab), device="cuda"), api.new_stats(n)
    ws = m.workspace(256, P)
    ws.view(torch.uint8).fill_(0xff)
    m.sb_verify_forward(k, v, P, torch.from_numpy(tokens).cuda(), parents, 1.0, logits, stats, ws)
    torch.cuda.synchronize()
    ref = int8.tree_forward(shape, W, K, V, P, tokens, parents)[0]
    check_logits(logits.cpu().numpy(), ref, decoder.tree_forward(shape, W, K, V, P, tokens, parents, "bf16")[0])


def test_forward_noalloc_and_timed(api):
    shape = synth.SHAPES["small_h128_bf16"]
    m = api.Model(shape, api.synth_tensors(shape), projections="int8")
    n, P = 9, 30
    k, v = m.new_kv(P + n)
    k.normal_()
    v.normal_()
    toks = torch.arange(n, dtype=torch.int32, device="cuda")
    a, b = torch.empty((n, shape.vocab), device="cuda"), torch.empty((n, shape.vocab), device="cuda")
    par = synth.fork_parents(0, 2, 4)
    m.sb_timer_start("gate_up", 8)
    m.sb_verify_forward(k, v, P, toks, par, 1.0, a, api.new_stats(n), m.workspace(n, P))
    ms, launches = m.sb_timer_stop()
    assert launches == shape.n_layers and ms > 0
    m.sb_verify_forward_noalloc(k, v, P, toks, par, 1.0, b, api.new_stats(n))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_forward_on_the_quantized_cache(api, form):
    """Both 8-bit forms together: projections and prefix."""
    shape, nb, tail = synth.SHAPES["small_gqa_bf16"], 2, 10
    W, parents = weights(shape), synth.fork_parents(1, 3, 3)
    n, P, g = len(parents), 64 * nb + tail, np.random.default_rng(5)
    m = api.Model(shape, api.dict_tensors(W), projections="int8")
    K = bf16(g.standard_normal((shape.n_layers, shape.n_kv_heads, P, shape.head_dim))).float().numpy()
    V = bf16(g.standard_normal(K.shape)).float().numpy()
    tokens = g.integers(0, shape.vocab, n).astype(np.int32)
    k, v = m.new_kv(P)
    m.load_kv(k, v, K, V, P)
    c = api.QuantizedKV(m.cfg, 64 * nb, tail + n, form)
    api.sb_kv_quantize(m.cfg, k, v, 0, c, 0, nb)
    c.tail_k[:, :, :tail], c.tail_v[:, :, :, :tail] = k[:, :, 64 * nb:P], v[:, :, :, 64 * nb:P]
    logits, stats = torch.empty((n, shape.vocab), device="cuda"), api.new_stats(n)
    m.sb_verify_forward_quantized(c, nb, tail, torch.from_numpy(tokens).cuda(), parents, 1.0, logits, stats,
                                  m.quantized_workspace(n, nb, tail))
    torch.cuda.synchronize()
    seen = [np.concatenate([quantized.values(*quantized.quantize(x[:, :, :64 * nb], form)), x[:, :, 64 * nb:]], 2)
            for x in (K, V)]
    ref, _, _ = int8.tree_forward(shape, W, *seen, P, tokens, parents)
    plain, _, _ = decoder.tree_forward(shape, W, *[x.astype(np.float32) for x in seen], P, tokens, parents, "bf16")
    check_logits(logits.cpu().numpy(), ref, plain)


def test_round_with_int8_models(api):
    """Algorithm 2's round takes int8 models as it takes bf16 ones: on two
    streams and on one, the same tokens, caches and lengths."""
    shape = synth.SHAPES["small_gqa_bf16"]
    tm = api.Model(shape, api.synth_tensors(shape, 0), projections="int8")
    dm = api.Model(shape, api.synth_tensors(shape, 1), projections="int8")
    P, params = 30, api.round_params(4, "wor", 3, 4, 0.0005, 1.0)
    nd, V = 4 + 4 * 3, shape.vocab
    g = torch.Generator(device="cuda").manual_seed(4)
    u = torch.rand(nd + 5 + 5, device="cuda", generator=g)
    outs = []
    for two in (True, False):
        gk = torch.Generator(device="cuda").manual_seed(9)
        caches = []
        for m in (tm, dm):
            k, v = m.new_kv(P + nd)
            k[:, :, :P] = torch.randn(k[:, :, :P].shape, device="cuda", generator=gk).bfloat16()
            v[:, :, :, :P] = torch.randn(v[:, :, :, :P].shape, device="cuda", generator=gk).bfloat16()
            caches.append((k, v))
        buf = api.RoundBuffers(tm, dm, params, P, P)
        buf.tokens[0] = 3
        torch.cuda.synchronize()
        sv = torch.cuda.Stream()
        sd = torch.cuda.Stream() if two else sv
        c, B, par = api.sb_spec_round(tm, *caches[0], P, dm, *caches[1], P, u[:nd], u[nd:nd + 5].contiguous(),
                                      u[nd + 5:].contiguous(), buf, sv, sd)
        torch.cuda.synchronize()
        r = api.decode_round(buf.round)
        assert 0 <= r["token"] < V and r["flags"] == 0
        outs.append((c, B, r, buf.new_lens.tolist(), buf.tokens[:1 + c + B * 3].tolist(), caches))
    assert outs[0][:5] == outs[1][:5]
    for (k0, v0), (k1, v1) in zip(outs[0][5], outs[1][5]):
        assert torch.equal(k0, k1) and torch.equal(v0, v1)
