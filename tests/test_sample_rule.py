"""The rule that tests of drawn tokens use: it takes the oracle's draws, and
refuses other tokens and the draws of oracles with a mistake in them."""
import numpy as np
import pytest

from oracle import chunk as orc
from sample_rule import Row, accepted

FILTERS = [dict(), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.9999), dict(min_p=0.05), dict(top_k=100, top_p=0.97, min_p=0.02)]


def row_of(V, seed, spread=2.0):
    l = (np.random.default_rng(seed).normal(size=V) * spread).astype(np.float32)
    l[V - V // 100:] = -np.inf
    return l


@pytest.mark.parametrize("V", [5, 1000, 151936])
@pytest.mark.parametrize("f", FILTERS, ids=str)
def test_the_oracles_token_and_no_other(V, f):
    rng = np.random.default_rng(V)
    f = {k: v if k == "top_k" else np.float32(v) for k, v in f.items()}
    for T in (1.0, 0.7, 3.0):
        l = row_of(V, 3 + V)
        row = Row(l, np.float32(T))
        for u in rng.random(3).astype(np.float32):
            token, lp = orc.sample(l, u, temperature=np.float32(T), **f)
            assert accepted(l, u, token, np.float32(lp), temperature=np.float32(T), row=row, **f) is None
            assert accepted(l, u, token, np.float32(lp * 1.001 + 0.001), temperature=np.float32(T), row=row, **f)
            ids, _ = orc.kept_tokens(l, temperature=np.float32(T), **f)
            at = int(np.nonzero(ids == token)[0][0])
            near = [int(ids[i]) for i in (at - 1, at + 1) if 0 <= i < len(ids)]
            for wrong in near + rng.integers(0, V, 5).tolist() + [-1, V, V - 1]:
                if wrong != token:
                    assert accepted(l, u, wrong, np.float32(lp), temperature=np.float32(T), row=row, **f), (wrong, token)


def test_the_longest_row():
    """2^20 equal-ish logits, where a token has a millionth of the mass."""
    V = 1 << 20
    l = row_of(V, 9)
    for f in (dict(), dict(top_p=np.float32(0.9))):
        token, lp = orc.sample(l, np.float32(0.4), temperature=3.0, **f)
        row = Row(l, 3.0)
        u = np.float32(0.4)
        assert accepted(l, u, token, lp, temperature=3.0, row=row, **f) is None
        for wrong in (-1, 0, token - 1, token + 1, V - 1):
            assert accepted(l, u, wrong, lp, temperature=3.0, row=row, **f)


def wrong_draw(mistake, l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The oracle's draw with one mistake."""
    l64 = l.astype(np.float64)
    order = np.argsort(-l64, kind="stable")
    if mistake == "ties by the highest index":
        order = order[np.lexsort((-order, -l64[order]))]
    order = order[l64[order] > -np.inf]
    w = np.exp((l64[order] - l64[order[0]]) / temperature)
    n = int(top_k) if top_k > 0 else len(order)
    keep = np.arange(len(order)) < n
    mass = w if mistake == "top-p of the whole row" else w[:n]
    before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
    want = float(top_p) * mass.sum()
    if top_p < 1.0:
        keep &= before + w < want if mistake == "top-p stops one early" else before < want
        keep[0] = True
    if mistake == "min-p of the total":
        keep &= w / w.sum() >= min_p
        keep[0] = True
    else:
        keep &= w >= min_p
    order, w = order[keep], w[keep]
    by_id = np.argsort(order)
    order, w = order[by_id], w[by_id]
    run = np.cumsum(w.astype(np.float32)).astype(np.float64) if mistake == "sums in 32 bits" else np.cumsum(w)
    total = w.sum() if mistake != "u times the unfiltered total" else np.exp((l64[l64 > -np.inf] - l64.max()) / temperature).sum()
    j = min(int(np.searchsorted(run, float(u) * total, side="right")), len(order) - 1)
    return int(order[j]), float(np.log(w[j] / w.sum()))


@pytest.mark.parametrize("mistake", ["none", "ties by the highest index", "top-p of the whole row", "top-p stops one early",
                                     "min-p of the total", "u times the unfiltered total", "sums in 32 bits"])
def test_mistakes_are_refused(mistake):
    f = dict(top_k=30, top_p=np.float32(0.9), min_p=np.float32(0.02))
    rows = [row_of(500, s, 1.0) for s in range(4)]
    if mistake == "ties by the highest index":
        rows = [np.round(l * 2) / 2 for l in rows]
    if mistake == "sums in 32 bits":
        f, rows = {}, [row_of(151936, s, 1.0) for s in range(4)]
    refused = 0
    for l in rows:
        row = Row(l, 1.0)
        for u in np.linspace(0.01, 0.99, 13, dtype=np.float32):
            token, lp = wrong_draw(mistake, l, u, **f)
            refused += accepted(l, u, token, lp, row=row, **f) is not None
    assert refused == 0 if mistake == "none" else refused > 0


def test_rows_without_a_draw():
    nothing = np.full(4, -np.inf, np.float32)
    assert accepted(nothing, 0.5, -1, -np.inf) is None and accepted(nothing, 0.5, 0, 0.0)
    l = np.array([1, 3, 3, -np.inf, np.nan], np.float32)
    assert accepted(l, 0.5, 1, 0.0, temperature=0.0) is None and accepted(l, 0.5, 2, 0.0, temperature=0.0)
    assert accepted(l, 0.9, 4, -1.0) and accepted(l, 0.9, 3, -1.0)
