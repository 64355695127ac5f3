"""Rules on logits (penalties, biases, masks) in float64 numpy.  For checking only.

TEST INFRASTRUCTURE ONLY: the product library never uses this module, and
nothing here is shared with it.
"""
from __future__ import annotations

import numpy as np


def _given(p, b, off, above=None):
    x = off if p is None else float(p[b])
    return off if not np.isfinite(x) or (above is not None and not x > above) else x


def row(l, b, tokens=None, lens=None, prompt_lens=None, repetition=None, frequency=None, presence=None,
        bias_starts=None, bias_tokens=None, bias_values=None, allowed=None):
    """(x, size): row b's logits l after its rules, and the largest magnitude met on
    the way (finite ones), the scale of rounding errors."""
    x = np.array(l, dtype=np.float64)
    size = np.where(np.isfinite(x), np.abs(x), 0.0)
    V = len(x)

    def met(y):
        return np.maximum(size, np.where(np.isfinite(y), np.abs(y), 0.0))

    with np.errstate(invalid="ignore", over="ignore"):
        if tokens is not None:
            n = min(max(int(lens[b]), 0), tokens.shape[1])
            p = 0 if prompt_lens is None else min(max(int(prompt_lens[b]), 0), n)
            ids = tokens[b, :n].astype(np.int64)
            known = (ids >= 0) & (ids < V)
            seen = np.unique(ids[known])
            r = _given(repetition, b, 1.0, above=0.0)
            x[seen] = np.where(x[seen] > 0, x[seen] / r, x[seen] * r)
            size = met(x)
            times = np.bincount(ids[p:][known[p:]], minlength=V)
            f, q = _given(frequency, b, 0.0), _given(presence, b, 0.0)
            size = np.maximum(size, np.where(times > 0, np.abs(f * times) + abs(q), 0.0))
            x = np.where(times > 0, x - (f * times + q), x)
            size = met(x)
        if bias_starts is not None:
            a, e = (min(max(int(bias_starts[i]), 0), len(bias_tokens)) for i in (b, b + 1))
            total, mass = np.zeros(V), np.zeros(V)
            for t, w in zip(bias_tokens[a:e], bias_values[a:e]):
                if 0 <= t < V:
                    total[t] += w
                    mass[t] += abs(w) if np.isfinite(w) else 0.0
            x = x + total
            size = np.maximum(met(x), mass)
        if allowed is not None:
            v = np.arange(V)
            bits = allowed[b].astype(np.int64)[v // 32] >> (v % 32) & 1
            x[bits == 0] = -np.inf
    return x, size
