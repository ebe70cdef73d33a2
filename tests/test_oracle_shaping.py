"""CPU pins of the logit rules' oracle, and the host checks of their entry
points (nothing here launches)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import shaping


def test_rules_by_hand():
    """One token at a time, in Python, over a tree whose paths differ."""
    g = np.random.default_rng(0)
    V, parents, tokens = 40, [-1, 0, 0, 1, 3], [7, 7, 9, 7, 39]
    logits = g.standard_normal((5, V)).astype(np.float32)
    prompt, output = shaping.count([1, 2, 2], V), shaping.count([7, 9, 7, 4], V)
    bias = g.standard_normal(V).astype(np.float32)
    mask = np.array([[0xffffffff, 0x7f]] * 5, np.uint32)
    mask[3] = [0xf0f0f0f0, 0x80]
    out = shaping.shape(logits, tokens, parents, prompt, output, 1.25, 0.5, 0.25, bias, mask, np.float64)
    paths = [[], [1], [2], [1, 3], [1, 3, 4]]
    for i in range(5):
        for v in range(V):
            c = [7, 9, 7, 4].count(v) + [tokens[j] for j in paths[i]].count(v)
            l = float(logits[i, v])
            if c or v in (1, 2):
                l = l / 1.25 if l > 0 else l * 1.25
            l -= 0.25 * c + (0.5 if c else 0.0)
            l += float(bias[v])
            if not (int(mask[i, v // 32]) >> (v % 32)) & 1:
                l = -np.inf
            assert out[i, v] == pytest.approx(l, rel=1e-14) or out[i, v] == l


def test_masks_hide_what_is_under_them():
    logits = np.array([[np.nan, np.inf, 1.0]], np.float32)
    out = shaping.shape(logits, [0], [-1], bias=np.array([0, 0, -np.inf], np.float32), mask=np.array([4], np.uint32))
    assert np.array_equal(out, [[-np.inf, -np.inf, -np.inf]])
    assert np.array_equal(shaping.count([-1, 5, 2, 2], 5), [0, 0, 2, 0, 0])


@pytest.fixture(scope="module")
def api():
    from paper_2506_01979_amd import api as A
    return A


def test_count_refusals(api):
    f = api.lib.sb_count_tokens
    assert f(0, 1, 16, 0, 16, None) == 1 and f(10, -1, 16, 0, 16, None) == 1
    assert f(10, 1, None, 0, 16, None) == 1 and f(10, 1, 16, 0, None, None) == 1
    assert f((1 << 20) + 1, 1, 16, 0, 16, None) == 1
    assert f(10, 0, None, 1, 16, None) == 0                      # nothing to add
    f = api.lib.sb_count_step
    assert f(0, 1, 16, 16, 16, None) == 1 and f(10, 0, 16, 16, 16, None) == 1 and f(10, 257, 16, 16, 16, None) == 1
    assert f(10, 1, None, 16, 16, None) == 1 and f(10, 1, 16, None, 16, None) == 1 and f(10, 1, 16, 16, None, None) == 1


def test_shape_refusals(api):
    par = (C.c_int32 * 3)(-1, 0, 1)
    need = api.sb_shape_workspace_bytes(1000, 3)

    def call(vocab=1000, n=3, toks=16, p=par, logits=16, out=16, T=1.0, stats=16, ws=16, size=need, **rules):
        f = dict(prompt=None, output=None, repetition=1.0, presence=0.0, frequency=0.0, bias=None, mask=None, stride=0)
        f.update(rules)
        return api.lib.sb_shape_logits(vocab, n, C.byref(api.LogitRulesStruct(*f.values())), toks, p, logits, out, T,
                                       stats, ws, size, None)
    assert call(vocab=0) == 1 and call(vocab=(1 << 20) + 1) == 1 and call(n=0) == 1 and call(n=257) == 1
    for k in ("toks", "logits", "out", "stats", "ws", "p"):
        assert call(**{k: None}) == 1
    assert call(ws=24) == 1
    assert call(p=(C.c_int32 * 3)(-1, 0, 2)) == 2
    assert call(T=-1.0) == 1 and call(T=float("inf")) == 1
    nan, inf = float("nan"), float("inf")
    for x in (0.0, -1.0, nan, inf):
        assert call(repetition=x) == 1
    for x in (nan, inf):
        assert call(presence=x) == 1 and call(frequency=x) == 1
    assert call(mask=16, stride=31) == 1 and call(mask=16, stride=-32) == 1   # 32 words a row
    assert call(size=need - 1) == 3
    assert api.lib.sb_shape_logits(1000, 3, None, 16, par, 16, 16, 1.0, 16, 16, need, None) == 1


@pytest.mark.parametrize("vocab", [1, 1000, 32000, 128256, 262145, 1 << 20])
def test_shape_workspace_serves_smaller_trees(api, vocab):
    sizes = [api.sb_shape_workspace_bytes(vocab, n) for n in range(1, 257)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert api.sb_shape_workspace_bytes(vocab, 0) == 0 and api.sb_shape_workspace_bytes(vocab, 257) == 0


def test_binding_refuses_other_shapes(api):
    with pytest.raises(ValueError, match="device"):
        api.LogitRules(bias=torch.zeros(10))
    with pytest.raises(ValueError, match="mask"):
        api.LogitRules(mask=torch.zeros(10, dtype=torch.int64))
