"""GPU parity of token counts and of the logit rules: counts and shaped logits
are the oracle's bit for bit (float32, every operation rounded on its own), the
statistics the oracle's of the same logits -- zmax and argmax exact, the total
within 1e-6 relative (float32 exponentials summed in float64)."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import sampling, shaping
from paper_2506_01979_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    assert torch.cuda.is_available()
    return A


def dev(x, dt=None):
    return torch.from_numpy(np.ascontiguousarray(x, dt)).cuda()


# ---- counts ------------------------------------------------------------------------

@pytest.mark.parametrize("vocab", [1, 5, 1024, 1025, 32000, 128256, 1 << 20])
@pytest.mark.parametrize("n", [0, 1, 33, 1024, 9001, 70000])
def test_count_tokens(api, vocab, n):
    g = np.random.default_rng(n + vocab)
    say("count", vocab, n)
    # mostly one token, some out of the vocabulary
    t = np.where(g.random(n) < 0.3, vocab // 2, g.integers(-3, vocab + 3, n)).astype(np.int32)
    counts = torch.full((vocab + 8,), 77, dtype=torch.int32, device="cuda")
    toks = dev(t, np.int32)
    api.sb_count_tokens(toks, counts[:vocab], accumulate=False)
    ref = shaping.count(t, vocab)
    assert np.array_equal(counts[:vocab].cpu().numpy(), ref)
    api.sb_count_tokens(toks[n // 2:], counts[:vocab])
    assert np.array_equal(counts[:vocab].cpu().numpy(), ref + shaping.count(t[n // 2:], vocab))
    assert (counts[vocab:] == 77).all()


def test_count_most_tokens(api):
    """2^31 - 1 tokens, none in the vocabulary but some of the last."""
    n = 2 ** 31 - 1
    t = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    t[-5000:-1] = 3
    counts = torch.ones(5, dtype=torch.int32, device="cuda")
    say("count most")
    api.sb_count_tokens(t, counts)
    assert counts.tolist() == [1, 1, 1, 5000, 1]


def test_count_step(api):
    V, toks = 50, [3, 4, 5, 4, 60, 6]
    for path, nxt, want in (([0, 1, 3], 7, [4, 4, 7]), ([0], 3, [3]), ([0, 4, 5], 4, [6, 4]),
                            ([0, 2], -1, [5]), ([0, 2, 9], 50, [5])):
        r = np.full(api.STEP_RESULT_INTS, -1, np.int32)
        r[0], r[2], r[3] = len(path) - 1, nxt, len(path)
        r[8:8 + len(path)] = path
        counts = torch.ones(V, dtype=torch.int32, device="cuda")
        api.sb_count_step(dev(toks, np.int32), dev(r), counts)
        assert np.array_equal(counts.cpu().numpy(), 1 + shaping.count(want, V)), path
    r = np.full(api.STEP_RESULT_INTS, 1, np.int32)      # a whole chain of 256 rows, all one token
    r[2], r[3], r[8:] = 9, 256, np.arange(256)
    counts = torch.zeros(V, dtype=torch.int32, device="cuda")
    api.sb_count_step(torch.full((256,), 9, dtype=torch.int32, device="cuda"), dev(r), counts)
    assert int(counts[9]) == 256 and int(counts.sum()) == 256


# ---- rules --------------------------------------------------------------------------

def case(g, V, parents, rep, pres, freq, bias, mask, history=300):
    n = len(parents)
    hot = g.integers(0, V, 12)                          # tokens that repeat
    pick = lambda k: np.where(g.random(k) < 0.5, hot[g.integers(0, 12, k)], g.integers(0, V, k)).astype(np.int32)  # noqa: E731
    x = dict(logits=(3 * g.standard_normal((n, V))).astype(np.float32), tokens=pick(n))
    r = dict(prompt=shaping.count(pick(history), V), output=shaping.count(pick(history // 2), V), repetition=rep,
             presence=pres, frequency=freq)
    if bias:
        b = np.where(g.random(V) < 0.2, 4 * g.standard_normal(V), 0).astype(np.float32)
        b[g.integers(0, V, 5)] = -np.inf
        b[g.integers(0, V, 3)] = np.finfo(np.float32).min
        r["bias"] = b
    if mask != "none":
        rows = n if mask == "rows" else 1
        share = g.random((rows, 1)) ** 2
        bits = g.random((rows, (V + 31) // 32, 32)) < share[..., None]
        r["mask"] = (bits.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return x, r


def rules_on_device(api, r):
    d = {k: (dev(v.view(np.int32) if k == "mask" else v) if isinstance(v, np.ndarray) else v) for k, v in r.items()}
    return api.LogitRules(**d)


def run(api, x, r, parents, T, out=None, shift=0):
    n, V = x["logits"].shape
    # shift: the logits' rows off 16-byte alignment
    buf = torch.empty(n * V + shift, device="cuda")[shift:].view(n, V)
    buf.copy_(dev(x["logits"]))
    out = buf if out == "in place" else torch.full((n + 1, V), 5.0, device="cuda")
    stats = api.new_stats(n)
    ws = torch.full((api.sb_shape_workspace_bytes(V, n),), 0xff, dtype=torch.uint8, device="cuda")
    api.sb_shape_logits(rules_on_device(api, r), dev(x["tokens"], np.int32), parents, buf, out, T, stats, ws)
    torch.cuda.synchronize()
    if out is not buf:
        assert (out[n] == 5.0).all()
    return out[:n].cpu().numpy(), api.decode_stats(stats)


def check(got, st, ref, T):
    assert np.array_equal(got, ref, equal_nan=True)
    for i in range(len(ref)):
        if np.all(ref[i] == -np.inf):
            assert np.isnan(st["total"][i]) and st["argmax"][i] == 0
            continue
        rs = sampling.row_stats(ref[i], T)
        assert st["argmax"][i] == rs.argmax and np.float32(st["zmax"][i]) == np.float32(rs.zmax), i
        if np.isnan(rs.total):
            assert np.isnan(st["total"][i])
        else:
            assert abs(st["total"][i] - rs.total) <= 1e-6 * rs.total, (i, st["total"][i], rs.total)


TREES = {"root": [-1], "chain5": [-1, 0, 1, 2, 3], "fork": synth.fork_parents(2, 3, 4), "chain256": list(range(-1, 255)),
         "wide": [-1] + [0] * 40}


@pytest.mark.parametrize("V", [1, 3, 32, 1000, 1001, 4096, 32000])
@pytest.mark.parametrize("tree", list(TREES))
@pytest.mark.parametrize("T", [0.0, 0.7, 1.0])
def test_all_rules(api, V, tree, T):
    parents = TREES[tree]
    g = np.random.default_rng(V + len(parents))
    say("shape", V, tree, T)
    x, r = case(g, V, parents, 1.3, 0.4, 0.15, True, "rows")
    got, st = run(api, x, r, parents, T)
    check(got, st, shaping.shape(x["logits"], x["tokens"], parents, **r), T)


@pytest.mark.parametrize("rep,pres,freq,bias,mask", [
    (1.0, 0.0, 0.0, False, "none"), (1.2, 0.0, 0.0, False, "none"), (0.8, 0.0, 0.0, False, "one"),
    (1.0, -0.5, 0.0, False, "none"), (1.0, 0.0, 0.25, True, "none"), (1.0, 0.0, 0.0, True, "one"),
    (1.0, 0.0, 0.0, False, "rows")])
@pytest.mark.parametrize("place", ["in place", "apart"])
@pytest.mark.parametrize("shift", [0, 1])
def test_each_rule(api, rep, pres, freq, bias, mask, place, shift):
    parents, V = synth.fork_parents(1, 2, 3), 2052
    g = np.random.default_rng(11)
    x, r = case(g, V, parents, rep, pres, freq, bias, mask)
    say("rule", rep, pres, freq, bias, mask, place, shift)
    got, st = run(api, x, r, parents, 1.0, place, shift)
    check(got, st, shaping.shape(x["logits"], x["tokens"], parents, **r), 1.0)
    r.update(prompt=None, output=None)                  # the drafts alone
    got, st = run(api, x, r, parents, 1.0, place, shift)
    check(got, st, shaping.shape(x["logits"], x["tokens"], parents, **r), 1.0)


@pytest.mark.parametrize("rep", [1.2, 0.75, 1 + 2 ** -23, 2 - 2 ** -22, 3e-7, 5e6, 1e-30, 1e30])
@pytest.mark.parametrize("tree", ["root", "chain256"])
def test_quotients(api, rep, tree):
    """Every size of a logit, zeros and subnormals among them, by repetitions near one and far
    from it: the quotients and products are the rounded ones."""
    parents, V = TREES[tree], 5004 if tree == "root" else 1001
    g = np.random.default_rng(21)
    x, r = case(g, V, parents, rep, 0.0, 0.0, False, "none", 4000)
    n = len(parents)
    x["logits"] = (g.standard_normal((n, V)) * np.exp(g.uniform(-6 if n > 1 else -100, 6 if n > 1 else 85, (n, V)))).astype(np.float32)
    x["logits"][0, ::7] = 0.0
    x["logits"][0, 1::7] = (g.standard_normal(len(x["logits"][0, 1::7])) * 1e-40).astype(np.float32)
    say("quotients", rep, tree)
    got, _ = run(api, x, r, parents, 1.0)
    with np.errstate(over="ignore"):
        ref = shaping.shape(x["logits"], x["tokens"], parents, **r)
    assert np.array_equal(got, ref)


@pytest.mark.parametrize("T", [0.0, 1.0])
def test_values_in_masked_places_and_empty_rows(api, T):
    parents, V = [-1, 0, 1, 1, 0], 1000
    g = np.random.default_rng(4)
    x, r = case(g, V, parents, 1.1, 0.2, 0.1, False, "rows")
    bits = np.unpackbits(r["mask"].view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool)
    bits[:, 17] = True
    bits[1] = False                                     # nothing left
    bits[2] = False
    bits[2, V - 1] = True                               # one token left, the last
    packed = np.zeros((5, 32 * 32), bool)
    packed[:, :V] = bits
    packed[:, V:] = True                                # bits past the vocabulary mean nothing
    r["mask"] = np.packbits(packed, axis=1, bitorder="little").view(np.uint32)
    x["logits"][~bits] = np.where(g.random((~bits).sum()) < 0.5, np.nan, np.inf)
    x["logits"][3, 17] = np.nan                         # an allowed NaN
    got, st = run(api, x, r, parents, T)
    ref = shaping.shape(x["logits"], x["tokens"], parents, **r)
    check(got, st, ref, T)
    assert np.isnan(st["total"][1]) and np.isnan(st["total"][3]) and st["argmax"][2] == V - 1
    assert np.isfinite(st["total"][[0, 2, 4]]).all()


def test_large_vocabulary_and_ties(api):
    """A million tokens (slices of 4096), equal maxima: the lowest index."""
    parents, V = [-1, 0, 0], 1 << 20
    g = np.random.default_rng(5)
    x, r = case(g, V, parents, 1.5, 0.0, 0.0, False, "none")
    x["logits"] = np.round(x["logits"])
    got, st = run(api, x, r, parents, 0.5)
    check(got, st, shaping.shape(x["logits"], x["tokens"], parents, **r), 0.5)


def test_captured(api):
    """Replays follow the counts and logits, with eager work between."""
    parents, V = synth.fork_parents(0, 4, 8), 32000
    g = np.random.default_rng(6)
    x, r = case(g, V, parents, 1.2, 0.3, 0.1, True, "one")
    n = len(parents)
    rules = rules_on_device(api, r)
    logits, toks = dev(x["logits"]), dev(x["tokens"])
    out, stats = torch.empty_like(logits), api.new_stats(n)
    ws = torch.empty(api.sb_shape_workspace_bytes(V, n), dtype=torch.uint8, device="cuda")
    more = dev(g.integers(0, V, 50), np.int32)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        api.sb_count_tokens(more, rules.tensors[1])
        api.sb_shape_logits(rules, toks, parents, logits, out, 0.8, stats, ws)
    for i in range(3):
        logits.copy_(torch.randn_like(logits) * 3)
        graph.replay()
        torch.cuda.synchronize()
        r["output"] = r["output"] + shaping.count(more.cpu().numpy(), V)
        ref = shaping.shape(logits.cpu().numpy(), x["tokens"], parents, **r)
        check(out.cpu().numpy(), api.decode_stats(stats), ref, 0.8)


def test_step_under_rules(api):
    """As a constrained step uses them: the forward's logits shaped, the walk on
    the result, the committed tokens counted for the next step.  Every emitted
    token is one the grammar of its row allows, and the walk is the oracle's on
    the shaped logits."""
    shape = synth.SHAPES["small_bf16"]
    m = api.Model(shape, api.synth_tensors(shape))
    parents = synth.fork_parents(1, 2, 3)
    n, V, P = len(parents), shape.vocab, 40
    g = np.random.default_rng(9)
    k, v = m.new_kv(P + 8 * n)
    k.normal_()
    v.normal_()
    output = torch.zeros(V, dtype=torch.int32, device="cuda")
    mask = (g.random((n, (V + 31) // 32, 32)) < 0.3)
    words = (mask.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    bits = mask.reshape(n, -1)[:, :V]
    rules = api.LogitRules(output=output, repetition=1.2, frequency=0.3, mask=dev(words.view(np.int32)))
    logits, stats, res = torch.empty((n, V), device="cuda"), api.new_stats(n), api.new_result()
    ws, sws = m.workspace(n, P + 7 * n), torch.empty(api.sb_sample_workspace_bytes(V), dtype=torch.uint8, device="cuda")
    rws = torch.empty(api.sb_shape_workspace_bytes(V, n), dtype=torch.uint8, device="cuda")
    new_len, kv_len, said = torch.zeros(1, dtype=torch.int32, device="cuda"), P, []
    root = 5
    for step in range(5):
        # drafts that the grammar allows, from a flat q over the allowed tokens
        toks = np.array([root] + [int(g.choice(np.nonzero(bits[parents[i]])[0])) for i in range(1, n)], np.int32)
        q = np.zeros((n, V), np.float32)
        for i in range(1, n):
            q[i] = bits[parents[i]] / bits[parents[i]].sum()
        u = g.random(n).astype(np.float32)
        m.sb_verify_forward(k, v, kv_len, dev(toks), parents, 1.0, logits, stats, ws)
        raw = logits.cpu().numpy()
        api.sb_shape_logits(rules, dev(toks), parents, logits, logits, 1.0, stats, rws)
        api.sb_accept_resample(dev(toks), parents, logits, stats, 1.0, dev(q), dev(u), res, sws)
        m.sb_kv_rollback(k, v, kv_len, res, new_len)
        api.sb_count_step(dev(toks), res, output)
        torch.cuda.synchronize()
        ref = shaping.shape(raw, toks, parents, output=shaping.count(said, V), repetition=1.2, frequency=0.3, mask=words)
        assert np.array_equal(logits.cpu().numpy(), ref)
        r = api.decode_result(res)
        o = sampling.accept_resample(toks, parents, ref, 1.0, q, u)
        assert r["path"] == list(o.path) and r["next_token"] == o.next_token and r["flags"] == 0
        assert bits[r["path"][-1], r["next_token"]]
        said += [int(toks[j]) for j in r["path"][1:]] + [r["next_token"]]
        assert np.array_equal(output.cpu().numpy(), shaping.count(said, V))
        root, kv_len = r["next_token"], int(new_len.item())


def test_serving_steps(api):
    """A request on 8-bit weights and cache: forward, rules, walk, rollback of the tail,
    counts and commit, step after step.  The shaped rows are the oracle's of the GPU's logits, the
    walk its walk on them, the counts those of what was said, and lengths follow."""
    shape = synth.SHAPES["small_gqa_bf16"]
    m = api.Model(shape, api.synth_tensors(shape), projections="int8")
    parents = synth.fork_parents(9, 2, 4)
    n, V = len(parents), shape.vocab
    g = np.random.default_rng(31)
    cache = api.QuantizedKV(m.cfg, 192, 64 + n, "int8")
    output, prompt = torch.zeros(V, dtype=torch.int32, device="cuda"), dev(shaping.count(g.integers(0, V, 50), V))
    rules = api.LogitRules(prompt=prompt, output=output, repetition=1.1, presence=0.1)
    logits, stats, res = torch.empty((n, V), device="cuda"), api.new_stats(n), api.new_result()
    ws, sws = m.quantized_workspace(n, 3, 63), torch.empty(api.sb_sample_workspace_bytes(V), dtype=torch.uint8, device="cuda")
    rws = torch.empty(api.sb_shape_workspace_bytes(V, n), dtype=torch.uint8, device="cuda")
    new_len, nb, tail, said, root = torch.zeros(1, dtype=torch.int32, device="cuda"), 0, 0, [], 5
    for step in range(24):
        toks = np.concatenate([[root], g.integers(0, V, n - 1)]).astype(np.int32)
        m.sb_verify_forward_quantized(cache, nb, tail, dev(toks), parents, 1.0, logits, stats, ws)
        raw = logits.cpu().numpy()
        api.sb_shape_logits(rules, dev(toks), parents, logits, logits, 1.0, stats, rws)
        q = torch.softmax(logits, -1)[np.maximum(parents, 0)].contiguous()
        u = (g.random(n) * (0.4 if step % 3 else 1.0)).astype(np.float32)
        api.sb_accept_resample(dev(toks), parents, logits, stats, 1.0, q, dev(u), res, sws)
        m.sb_kv_rollback(cache.tail_k, cache.tail_v, tail, res, new_len)
        api.sb_count_step(dev(toks), res, output)
        torch.cuda.synchronize()
        ref = shaping.shape(raw, toks, parents, prompt=prompt.cpu().numpy(), output=shaping.count(said, V),
                            repetition=1.1, presence=0.1)
        assert np.array_equal(logits.cpu().numpy(), ref)
        r = api.decode_result(res)
        o = sampling.accept_resample(toks, parents, ref, 1.0, q.cpu().numpy(), u)
        assert r["path"] == list(o.path) and r["next_token"] == o.next_token and r["flags"] == 0
        said += [int(toks[j]) for j in r["path"][1:]] + [r["next_token"]]
        assert np.array_equal(output.cpu().numpy(), shaping.count(said, V))
        root = r["next_token"]
        nb, tail = api.sb_kv_commit(m.cfg, cache, nb, int(new_len.item()))
        assert 64 * nb + tail == len(said) and tail < 64
        say("serving step", step, nb, tail)
        if nb == 2:
            break
    assert nb >= 1


def test_captured_large_tree(api):
    """A tree of more than 128 rows, whose paths stand in the workspace, replayed beside eager calls
    for other trees on a workspace of their own."""
    V, parents = 1500, [-1] + [i // 2 for i in range(199)]
    n, g = len(parents), np.random.default_rng(17)
    x, r = case(g, V, parents, 1.2, 0.2, 0.1, False, "none")
    rules, toks, logits = rules_on_device(api, r), dev(x["tokens"], np.int32), dev(x["logits"])
    out, stats = torch.zeros((n, V), device="cuda"), api.new_stats(n)
    ws, ws2 = (torch.empty(api.sb_shape_workspace_bytes(V, 256), dtype=torch.uint8, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.sb_shape_logits(rules, toks, parents, logits, out, 1.0, stats, ws)
    for i in range(3):
        toks.copy_(dev(g.integers(0, V, n), np.int32) if i else toks)
        other, st2 = torch.zeros((n, V), device="cuda"), api.new_stats(n)
        api.sb_shape_logits(rules, toks, list(range(-1, n - 1)), logits, other, 1.0, st2, ws2)
        graph.replay()
        torch.cuda.synchronize()
        t = toks.cpu().numpy()
        check(out.cpu().numpy(), api.decode_stats(stats), shaping.shape(x["logits"], t, parents, **r), 1.0)
        check(other.cpu().numpy(), api.decode_stats(st2), shaping.shape(x["logits"], t, list(range(-1, n - 1)), **r), 1.0)
