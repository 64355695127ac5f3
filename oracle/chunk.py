"""Operators on packed rows in float64 numpy: attention of chunks of new tokens
over the paged cache, head norms with position rotation and append, and
sampling.  For checking only.

TEST INFRASTRUCTURE ONLY: the product library never uses this module, and
nothing here is shared with it.

Packed rows: sequence b owns rows starts[b] .. starts[b + 1] - 1, and ctx[b]
counts them, so its row i is at position ctx[b] - Q + i.  Starts are clamped to
the rows, lengths to what the page table has room for, in both operators.
"""
from __future__ import annotations


import numpy as np


def _length(ctx, b, table, page):
    return min(max(int(ctx[b]), 0), table.shape[1] * page)


def _owned(starts, b, rows):
    a, e = (min(max(int(x), 0), rows) for x in (starts[b], starts[b + 1]))
    return a, max(e, a)


def gather(pages, table_row, n, g):
    """The first n rows of head g of a sequence, in float64 (page ids outside
    the pool read as zeros)."""
    P, D = pages.shape[2], pages.shape[3]
    out = np.zeros((n, D))
    for j in range((n + P - 1) // P):
        pid = int(table_row[j])
        if 0 <= pid < pages.shape[0]:
            m = min(P, n - j * P)
            out[j * P:j * P + m] = pages[pid, g, :m]
    return out


def chunk_attention(q, k_pages, v_pages, table, ctx, starts, scale):
    """(out, mean |v|): out[r][h] = sum over visible keys of softmax * V, and the
    same sum of |V| (finite values only), the scale of its rounding errors.  Rows
    of no sequence come back as NaN in both.  Invisible values never enter."""
    T, Hq, D = q.shape
    Hkv = k_pages.shape[1]
    G = Hq // Hkv
    out, mag = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    for b in range(len(ctx)):
        a, e = _owned(starts, b, T)
        Q, L = e - a, _length(ctx, b, table, k_pages.shape[2])
        if Q == 0:
            continue
        last = np.arange(L - Q, L)                     # position of each row
        for g in range(Hkv):
            K, V = gather(k_pages, table[b], L, g), gather(v_pages, table[b], L, g)
            odd = ~np.isfinite(V)
            V0 = np.where(odd, 0.0, V)
            for h in range(g * G, (g + 1) * G):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (q[a:e, h].astype(np.float64) @ K.T)
                seen = np.arange(L)[None, :] <= last[:, None]
                s = np.where(seen, s, -np.inf)
                top = s.max(axis=1, keepdims=True) if L else np.zeros((Q, 1))
                with np.errstate(invalid="ignore"):
                    w = np.exp(s - np.where(np.isneginf(top), 0.0, top))
                    z = w.sum(axis=1, keepdims=True)
                    w = np.where(z == 0.0, 0.0, w / np.where(z == 0.0, 1.0, z))
                o = w @ V0
                for t, d in zip(*np.nonzero(odd)):
                    with np.errstate(invalid="ignore"):
                        o[seen[:, t], d] += w[seen[:, t], t] * V[t, d]
                out[a:e, h], mag[a:e, h] = o, w @ np.abs(V0)
    return out, mag


def rope_append(q, k, v, k_pages, v_pages, table, ctx, starts, inv_freq, q_norm=None, k_norm=None, eps=1e-6,
                interleaved=False):
    """(q_out, k_pages, v_pages) in float64; rows of no sequence are NaN in q_out,
    pages keep what no row writes."""
    T, Hq, D = q.shape
    P = k_pages.shape[2]
    f = np.asarray(inv_freq, dtype=np.float64)
    half = len(f)
    q_out = np.full(q.shape, np.nan)
    kp, vp = k_pages.astype(np.float64), v_pages.astype(np.float64)

    def turn(x, w, pos):
        x = x.astype(np.float64)
        if w is not None:
            x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * w.astype(np.float64)
        y = x.copy()
        first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
        second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
        c, s = np.cos(pos * f), np.sin(pos * f)
        y[:, first] = x[:, first] * c - x[:, second] * s
        y[:, second] = x[:, second] * c + x[:, first] * s
        return y

    for b in range(len(ctx)):
        a, e = _owned(starts, b, T)
        for r in range(a, e):
            pos = _length(ctx, b, table, P) - (e - r)
            q_out[r] = turn(q[r], q_norm, pos)
            if pos < 0:
                continue
            pid = int(table[b][pos // P])
            if 0 <= pid < k_pages.shape[0]:
                kp[pid, :, pos % P] = turn(k[r], k_norm, pos)
                vp[pid, :, pos % P] = v[r]
    return q_out, kp, vp


def kept_tokens(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token ids in ascending order, their float64 weights): what the filters
    leave of a row, weights relative to the largest logit's.  Unusable logits
    (-inf, NaN) are never kept."""
    l = np.asarray(logits, dtype=np.float64)
    ids = np.nonzero(l > -np.inf)[0]
    if len(ids) == 0:
        return ids, np.zeros(0)
    l = np.minimum(l, np.finfo(np.float32).max)
    order = ids[np.argsort(-l[ids], kind="stable")]       # equal logits: the lowest index first
    top = l[order[0]]
    if not temperature > 0.0:
        return order[:1], np.ones(1)
    w = np.exp((l[order] - top) / float(temperature))
    n = len(order) if top_k <= 0 else min(int(top_k), len(order))
    w = w[:n]
    keep = np.ones(n, dtype=bool)
    if 0.0 < min_p:
        keep &= w >= min(float(min_p), 1.0)
    if top_p < 1.0:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        keep &= before < max(float(top_p), 0.0) * w.sum()
        keep[0] = True
    order, w = order[:n][keep], w[keep]
    by_id = np.argsort(order)
    return order[by_id], w[by_id]


def sample(logits, u, **filters):
    """(token, log probability): the smallest kept token whose running weight in
    index order exceeds u times the total; (-1, -inf) if no logit is usable."""
    ids, w = kept_tokens(logits, **filters)
    if len(ids) == 0:
        return -1, -np.inf
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    run = np.cumsum(w)
    j = min(int(np.searchsorted(run, u * run[-1], side="right")), len(ids) - 1)
    return int(ids[j]), float(np.log(w[j] / run[-1]))


def border(logits, u, **filters):
    """How far the draw is from another token, in units of the total (a test that
    asks for equal tokens needs this above the rounding of either side)."""
    ids, w = kept_tokens(logits, **filters)
    run = np.cumsum(w) / w.sum()
    return float(np.abs(run[:-1] - float(u)).min()) if len(ids) > 1 else 1.0


