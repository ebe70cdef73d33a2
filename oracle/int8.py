"""Oracle of the 8-bit projections and of the forward on them (test
infrastructure only).

A row of x (a token) or of W (an output channel) with largest magnitude amax:
  scale = float32(amax / 127),  code = nearest(127 x / amax), ties to even
(amax = 0: scale 0; a NaN or infinity in the row: scale NaN, codes 0), and
  y[t][r] = sum_k code_x[t][k] code_w[r][k] * (scale_t scale_r).

``tree_forward`` is the decoder of oracle.decoder with these projections: the
input of each is quantised per token from the factored norm's h g (r = 1 / rms
multiplies afterwards), from the attention's output rounded to bfloat16, or from
silu(gate) up; q and k after RoPE, and v, are rounded to bfloat16.
"""
from __future__ import annotations

import numpy as np

from . import decoder, tree


def quantize(x: np.ndarray, dt=np.float64):
    """Codes and float32 scales of the rows of x.  dt float32: 127 x and the
    quotient each rounded to float32, as for float32 activations (to 24 bits also
    where 127 x is past float32: rows of such values are taken at 2^-16)."""
    x = np.asarray(x, dt)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        amax = np.abs(x).max(-1, keepdims=True)
        ok = np.isfinite(amax)
        scale = np.where(ok, amax.astype(np.float32) / np.float32(127), np.float32(np.nan))
        down = np.where(amax >= dt(2.0 ** 100), dt(2.0 ** -16), dt(1))
        codes = np.where(ok & (amax > 0), np.rint(x * down * dt(127) / (amax * down)), 0)
    return codes.astype(np.float64), scale[..., 0].astype(np.float32)


def linear(x: np.ndarray, w: np.ndarray, dt=np.float64) -> np.ndarray:
    """float32 y, rounded as the product is: the sum, the scales' product, theirs."""
    cx, sx = quantize(x, dt)
    cw, sw = quantize(w)
    return (cx @ cw.T).astype(np.float32) * (sx[:, None] * sw[None, :])


def tree_forward(shape, weights, prefix_k, prefix_v, kv_len, tokens, parents, hidden=None,
                 project=None, store=None):
    """As decoder.tree_forward.  project(x, w) and store(x) replace the product
    and the bfloat16 rounding (for the pins of this function)."""
    f8 = np.float64
    if project is None:
        memo = {}

        def project(x, w):
            cx, sx = quantize(x.astype(np.float32))
            if id(w) not in memo:
                memo[id(w)] = quantize(w)
            cw, sw = memo[id(w)]
            return (cx @ cw.T) * sx[:, None].astype(f8) * sw[None, :].astype(f8)
    if store is None:
        def store(x):
            return decoder.round_bf16(x.astype(np.float32)).astype(f8)
    parents = np.asarray(parents, np.int64)
    N, nh, nkv, d = len(tokens), shape.n_heads, shape.n_kv_heads, shape.head_dim
    cos, sin = decoder.rope_tables(kv_len + tree.depths(parents), d, shape.rope_theta, f8)
    paths = [tree.root_path(parents, i) for i in range(N)]

    def norm_project(h, gain, w):
        return project(h * np.asarray(gain, f8), w) * decoder.rms_scale(h, shape.rms_eps, f8)
    h = weights["embed"][np.asarray(tokens, np.int64)].astype(f8)
    k_tree = np.zeros((shape.n_layers, nkv, N, d))
    v_tree = np.zeros_like(k_tree)
    for li in range(shape.n_layers):
        W = weights["layers"][li]
        q = store(decoder.apply_rope(norm_project(h, W["attn_norm"], W["wq"]).reshape(N, nh, d), cos, sin))
        k = store(decoder.apply_rope(norm_project(h, W["attn_norm"], W["wk"]).reshape(N, nkv, d), cos, sin))
        v = store(norm_project(h, W["attn_norm"], W["wv"]).reshape(N, nkv, d))
        k_tree[li], v_tree[li] = k.transpose(1, 0, 2), v.transpose(1, 0, 2)
        o = np.zeros((N, nh, d))
        for i in range(N):
            for hh in range(nh):
                g = hh * nkv // nh
                K, V = k[paths[i], g], v[paths[i], g]
                if kv_len:
                    K = np.concatenate([np.asarray(prefix_k[li][g][:kv_len], f8), K])
                    V = np.concatenate([np.asarray(prefix_v[li][g][:kv_len], f8), V])
                s = K @ q[i, hh] / np.sqrt(d)
                p = np.exp(s - s.max())
                o[i, hh] = (p / p.sum()) @ V
        h = h + project(store(o.reshape(N, nh * d)), W["wo"])
        gate, up = norm_project(h, W["mlp_norm"], W["wg"]), norm_project(h, W["mlp_norm"], W["wu"])
        h = h + project(decoder.silu(gate) * up, W["wd"])
        if hidden is not None:
            hidden.append(h.copy())
    return norm_project(h, weights["final_norm"], weights["lm_head"]), k_tree, v_tree
