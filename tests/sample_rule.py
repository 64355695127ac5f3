"""Which tokens a draw may return.  A rule for tests: unlike "the oracle's token,
or anything where the draw is close to a border", it asks of the drawn token
itself that it is kept, that the running mass of the kept tokens passes u times
their total inside it, and that its log probability is its own.

How far masses may be off.  In units of the largest weight, a unit is at most
U = 2^-41.5 (2^-42 of a power of two that is at most a factor of sqrt(2) above the
largest weight or below it).  The polynomial of a weight w is off by at most 1.48
units of its own power of two, so by 2.1 U w (sqrt(2) for that power); the shift to
the row's unit takes at most min(U, w); sums of slices and of bins are shifted
once more, each by less than a unit and less than what they hold, which is at most
min(U, w) for each weight in them, at the filter and at the draw.  The exponent
l / T is rounded at its own size (2^-53 |l / T| of w), and 1 / T twice (2^-52 of
the distance from the largest logit).  So all masses of a row together are off by
at most
    S = sum_v (2.1 U + 2^-53 |l_v / T| + 2^-52 |l_v - max l| / T) w_v + 3 min(U, w_v),
and a comparison of two of them (a running mass and a fraction of a total) by 2 S.
Extended precision sums V weights to V 2^-64 of their total.
"""
import numpy as np

U = 2.0 ** -41.5
MIN_P_TOL = 2.0 ** -44   # log2(min_p) and (l - max l) log2(e) / T: three roundings of 2^-52 on at most 40 binary orders


class Row:
    """A row's usable logits in descending order (equal ones: the lowest index
    first), weights relative to the largest."""

    def __init__(self, logits, temperature):
        l = np.asarray(logits, dtype=np.float64)
        ids = np.nonzero(l > -np.inf)[0]
        l = np.minimum(l, np.finfo(np.float32).max)
        self.ids = ids[np.argsort(-l[ids], kind="stable")]
        if len(ids) == 0 or not temperature > 0.0:
            return
        x = l[self.ids].astype(np.longdouble)
        T = np.longdouble(temperature)
        z = (x - x[0]) / T
        self.w = np.exp(z)
        off = (2.1 * U + 2.0 ** -53 * np.abs(x / T) + 2.0 ** -52 * np.abs(z)) * self.w + 3 * np.minimum(U, self.w)
        self.slack = 2 * off.sum() + len(ids) * 2.0 ** -63 * self.w.sum()
        self.x_off = float(2.0 ** -52 * np.abs(x / T).max())


def accepted(logits, u, token, logprob, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, row=None):
    """None if the draw may return `token` with `logprob`, else what is wrong."""
    r = row or Row(logits, temperature)
    if len(r.ids) == 0:
        return None if token == -1 and logprob == -np.inf else "nothing to draw from"
    if not temperature > 0.0:
        return None if token == r.ids[0] and logprob == 0.0 else "not the largest logit"
    rank = np.nonzero(r.ids == token)[0]
    if len(rank) == 0:
        return "not a usable token"
    rank = int(rank[0])
    V = len(np.asarray(logits))
    k = min(int(top_k), len(r.ids)) if 0 < top_k < V else len(r.ids)
    w = r.w[:k]
    counts = {k}
    if top_p < 1.0:
        before = np.concatenate((np.zeros(1, np.longdouble), np.cumsum(w)[:-1]))
        want = np.longdouble(max(float(top_p), 0.0)) * w.sum()
        low, high = (max(1, int(np.searchsorted(before, want + d, side="left"))) for d in (-r.slack, r.slack))
        # between the two the kept mass grows by less than 2 slacks, but for the last one
        counts = {low, min(max(low, rank + 1), high), high}
    u = np.longdouble(min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0)
    wrong = "not kept"
    for n in counts:
        for tol in (-MIN_P_TOL, MIN_P_TOL):
            kept = np.ones(n, dtype=bool) if not min_p > 0.0 else w[:n] >= min(float(min_p), 1.0) * (1 - np.longdouble(tol))
            kept[0] = True
            if rank >= n or not kept[rank]:
                continue
            slack = r.slack * (2 if top_p < 1.0 else 1)
            mass = np.where(kept, w[:n], 0)
            total = mass.sum()
            start = mass[r.ids[:n] < token].sum()
            if start - slack > u * total or start + mass[rank] + slack <= u * total:
                wrong = f"the running mass passes u outside it: [{float(start / total)}, {float((start + mass[rank]) / total)}), u {float(u)}"
                continue
            lp = float(np.log(mass[rank] / total))
            if not abs(float(logprob) - lp) <= 2.0 ** -23 * abs(lp) + float(slack / total) + r.x_off + 2.0 ** -48:
                wrong = f"log probability {logprob} for {lp}"
                continue
            return None
    return wrong
