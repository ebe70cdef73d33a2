"""Oracle of the 8-bit prefix cache (test infrastructure only).

A block is 64 consecutive tokens of one (layer, KV head), of K or V.  With
amax the largest magnitude in it and top = 127 (int8) or 448 (e4m3: 4 exponent
bits with bias 7, 3 mantissa bits, largest 448):

  scale = float32(amax / top),  code = the nearest value of the type to
  x top / amax (ties to even),  value = code scale;

amax = 0 gives scale 0, a NaN or infinity in the block a NaN scale.  Everything
here is float64 but the scale, which the cache stores as float32.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
TOP = {"int8": 127.0, "e4m3": 448.0}


def nearest(y: np.ndarray, form: str) -> np.ndarray:
    """The value of the type nearest to y (|y| <= top), ties to even."""
    y = np.asarray(y, np.float64)
    if form == "int8":
        return np.rint(y)
    # |y| in [2^e, 2^(e+1)) has steps of 2^(e-3), e no less than -6 (subnormals)
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(y / step) * step


def quantize(x: np.ndarray, form: str):
    """x [..., n, d] with n a multiple of 64 -> (codes [..., n / 64, 64, d],
    scales float32 [..., n / 64])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-2], x.shape[-2] // BLOCK, BLOCK, x.shape[-1])
    with np.errstate(invalid="ignore", divide="ignore"):
        amax = np.abs(b).max((-2, -1))
        scales = np.where(np.isfinite(amax), amax / TOP[form], np.nan).astype(np.float32)
        live = np.isfinite(amax) & (amax > 0)
        y = b * TOP[form] / amax[..., None, None]
        codes = np.where(live[..., None, None], nearest(np.where(live[..., None, None], y, 0.0), form), 0.0)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """[..., nb, 64, d], [..., nb] -> [..., 64 nb, d]: what the cache stands for."""
    v = codes * scales.astype(np.float64)[..., None, None]
    return v.reshape(*v.shape[:-3], -1, v.shape[-1])


def commit(codes, scales, tail: np.ndarray, tail_len: int, form: str):
    """The tail's full blocks behind the codes, the rest at its front: (codes,
    scales, tail, tail_len)."""
    full = tail_len // BLOCK
    c, s = quantize(tail[..., :full * BLOCK, :], form)
    out = tail.copy()
    rest = tail_len - full * BLOCK
    if full:
        out[..., :rest, :] = tail[..., full * BLOCK:tail_len, :]
    return (np.concatenate([codes, c], -3), np.concatenate([scales, s], -1), out, rest)


def attend(q, k, v, paths):
    """q [n][heads][d]; k, v [n_kv][prefix + n][d] (the n tree rows last);
    paths bool [n][n]: row j on row i's path.  Returns the attention output
    [n][heads][d] and sum_j p_j |v_j|, the size its rounding errors scale
    with."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, nh, d = q.shape
    prefix = k.shape[1] - n
    seen = np.concatenate([np.ones((n, prefix), bool), paths], 1)
    out, size = np.empty_like(q), np.empty_like(q)
    for h in range(nh):
        g = h * k.shape[0] // nh
        s = np.where(seen, q[:, h] @ k[g].T / np.sqrt(d), -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[:, h] = p @ v[g]
        size[:, h] = p @ np.abs(v[g])
    return out, size
