"""Every drawn token is one that the rule of sample_rule.py allows: kept, with
the draw inside its own part of the running mass, and its own log probability.
Long vocabularies, filters that end in the tail, rows so flat that one bin holds
more than the list of candidates, and logits far from zero."""
import numpy as np
import pytest

from gpu_util import say
from sample_rule import Row, accepted
from test_gpu_sample import FILTERS, draw, logits_of

pytestmark = pytest.mark.gpu


def check(x, u, tag, temperature, f, rows=None):
    tokens, logprobs = draw(x, u, temperature=temperature, **{k: [v] * len(u) for k, v in f.items()})
    values = x.float().cpu().numpy()
    T = np.asarray(temperature, dtype=np.float32)
    rows = rows if rows is not None else [Row(values[b], T[b]) for b in range(len(u))]
    given = {k: v if k == "top_k" else np.float32(v) for k, v in f.items()}
    for b in range(len(u)):
        wrong = accepted(values[b], u[b], tokens[b], logprobs[b], temperature=T[b], row=rows[b], **given)
        assert wrong is None, f"{tag}: row {b} drew {tokens[b]} ({f}, T {T[b]}, u {u[b]}): {wrong}"
    return rows


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [1000, 50257, 151936, 1 << 20])
def test_every_filter(V, dtype):
    rng = np.random.default_rng(V + 1)
    T = [1.0, 0.7, 3.0, 0.2] if V < 1 << 20 else [1.0, 3.0]
    x = logits_of(len(T), V, dtype, 5 + V)
    rows = None
    for name, f in FILTERS.items():
        say("strict", V, dtype, name)
        rows = check(x, rng.random(len(T)).astype(np.float32), f"V {V} {dtype} {name}", T, f, rows)


@pytest.mark.parametrize("spread", [0.05, 0.4])
def test_flat_rows(spread):
    V = 151936
    x = logits_of(3, V, "float32", 31, spread=spread)
    rows = None
    for f in (dict(top_p=0.5), dict(top_p=0.99), dict(top_k=20000), dict(top_k=20000, top_p=0.7), dict(top_p=0.9, min_p=0.3),
              dict(top_k=9000, min_p=0.9)):
        say("flat", spread, f)
        rows = check(x, np.array([0.03, 0.5, 0.97], np.float32), f"spread {spread} {f}", [1.0] * 3, f, rows)


@pytest.mark.parametrize("offset, T", [(1e4, 1.0), (-1e4, 1.0), (0.0, 1e-3), (3e5, 0.5), (-1e3, 1e-3)])
def test_logits_far_from_zero(offset, T):
    """A common offset and a low temperature make l / T large, at whose size the
    exponent is rounded."""
    for V in (300, 50257):
        x = logits_of(4, V, "float32", 41, spread=2.0 if T > 0.1 else 2e-3)
        x = (x + offset).contiguous()
        rows = None
        for name, f in FILTERS.items():
            say("far", offset, T, V, name)
            rows = check(x, np.array([0.0, 0.35, 0.8, 0.99999], np.float32), f"offset {offset} T {T} V {V} {name}", [T] * 4, f, rows)
