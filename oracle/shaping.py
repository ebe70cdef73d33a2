"""Oracle of the rules on a token tree's logits (test infrastructure only).

Row i's history is the prompt's and the output's counts (the root among the
committed tokens) and the drafts on its path, rows 1 .. i.  With c = the
output's count plus those drafts, in float32, every operation rounded:

  seen (c > 0 or prompt > 0):  l = l > 0 ? l / repetition : l * repetition
  l = l - frequency c;  c > 0: l = l - presence;  l = l + bias
  a token whose mask bit is 0: -inf, whatever l was
"""
from __future__ import annotations

import numpy as np

from . import tree


def count(tokens, vocab: int) -> np.ndarray:
    t = np.asarray(tokens, np.int64)
    return np.bincount(t[(t >= 0) & (t < vocab)], minlength=vocab).astype(np.int32)


def allowed(mask, row: int, vocab: int) -> np.ndarray:
    """Bit v % 32 of word v / 32 of the row's mask (one mask serves all rows)."""
    words = np.atleast_2d(np.asarray(mask)).view(np.uint32)
    words = words[row if len(words) > 1 else 0]
    v = np.arange(vocab)
    return ((words[v // 32] >> (v % 32).astype(np.uint32)) & 1).astype(bool)


def shape(logits, tokens, parents, prompt=None, output=None, repetition=1.0, presence=0.0,
          frequency=0.0, bias=None, mask=None, dt=np.float32) -> np.ndarray:
    out = np.array(logits, dtype=dt)
    n, vocab = out.shape
    rep, pres, freq = (dt(np.float32(x)) for x in (repetition, presence, frequency))
    zero = np.zeros(vocab, np.int32)
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(n):
            path = [j for j in tree.root_path(np.asarray(parents), i) if j >= 1]
            c = (zero if output is None else output) + count([tokens[j] for j in path], vocab)
            seen = (c > 0) | ((zero if prompt is None else prompt) > 0)
            l = out[i]
            l = np.where(seen, np.where(l > 0, l / rep, l * rep), l)
            l = l - freq * c.astype(dt)
            l = np.where(c > 0, l - pres, l)
            if bias is not None:
                l = l + np.asarray(bias, dt)
            if mask is not None:
                l = np.where(allowed(mask, i, vocab), l, -np.inf)
            out[i] = l
    return out
