"""GPU tests of sampling against oracle/chunk.py in float64.

Tokens have to be equal unless the draw lies within rounding of a border:
weights are integers in units of 2^-42 of the largest, each off by at most one
unit, so a running sum of V of them, over a total of at least one largest
weight, is off by at most V 2^-42; 4 V 2^-42 covers both sides of a border and
the border of a top-p.  The log probability is rounded to float32 (2^-24
relative) and its total is off by at most V 2^-42.
"""
import numpy as np
import pytest

from oracle import chunk as orc
from gpu_util import say

pytestmark = pytest.mark.gpu


def draw(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, **kw):
    """Tokens and log probabilities; parameters are per-row lists or None."""
    import torch
    from paper_2608_22788_amd import binding
    B = logits.shape[0]
    vec = lambda x, dt: None if x is None else torch.tensor(np.asarray(x), dtype=dt, device="cuda")  # noqa: E731
    token = torch.full((B + 2,), -77, dtype=torch.int32, device="cuda")
    logprob = torch.full((B + 2,), 77.0, device="cuda")
    binding.sample(logits, vec(u, torch.float32), token[1:-1], logprob[1:-1], temperature=vec(temperature, torch.float32),
                   top_k=vec(top_k, torch.int32), top_p=vec(top_p, torch.float32), min_p=vec(min_p, torch.float32), **kw)
    torch.cuda.synchronize()
    t, lp = token.cpu().numpy(), logprob.cpu().numpy()
    assert t[0] == t[-1] == -77 and lp[0] == lp[-1] == 77.0
    return t[1:-1], lp[1:-1]


def check(logits, u, tag, **params):
    say(tag)
    tokens, logprobs = draw(logits, u, **params)
    values = logits.float().cpu().numpy()
    V = values.shape[1]
    slack = 4 * V * 2.0 ** -42
    for b in range(values.shape[0]):
        f = {k: np.float32(v[b]) if k != "top_k" else v[b] for k, v in params.items() if v is not None}
        want, lp = orc.sample(values[b], np.float32(u[b]), **f)
        if tokens[b] != want:
            near = min(orc.border(values[b], np.float32(u[b]), **f), top_p_border(values[b], f))
            assert near < slack, f"{tag}: row {b} drew {tokens[b]} instead of {want}, {near:g} from a border ({f}, u {u[b]})"
            continue
        if want < 0:
            assert logprobs[b] == -np.inf
        else:
            assert abs(logprobs[b] - lp) <= 2.0 ** -23 * abs(lp) + slack, f"{tag}: row {b} log prob {logprobs[b]} for {lp}"


def top_p_border(row, f):
    """Distance of p from the running masses that it is compared with."""
    if f.get("top_p", 1.0) >= 1.0:
        return 1.0
    g = {k: v for k, v in f.items() if k in ("temperature", "top_k")}
    _, w = orc.kept_tokens(row, **g)
    w = np.sort(w)[::-1]
    return float(np.abs(np.cumsum(w) / w.sum() - float(f["top_p"])).min())


def logits_of(B, V, dtype, seed, spread=2.0, holes=True):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(B, V, device="cuda").normal_(generator=g) * spread
    if holes and V > 8:
        x[torch.rand(B, V, generator=g, device="cuda") < 0.1] = -float("inf")
        x[:, V - V // 100:] = -float("inf")
    return x.to(getattr(torch, dtype))


FILTERS = {
    "none": {}, "k1": dict(top_k=1), "k40": dict(top_k=40), "k_many": dict(top_k=6000), "k_all": dict(top_k=1 << 20),
    "p": dict(top_p=0.9), "p_small": dict(top_p=1e-4), "p_most": dict(top_p=0.9999), "p_zero": dict(top_p=0.0),
    "m": dict(min_p=0.05), "m1": dict(min_p=1.0), "m_tiny": dict(min_p=1e-9),
    "kp": dict(top_k=50, top_p=0.8), "kp_many": dict(top_k=9000, top_p=0.95), "km": dict(top_k=30, min_p=0.2),
    "pm": dict(top_p=0.95, min_p=0.01), "kpm": dict(top_k=100, top_p=0.97, min_p=0.02)}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [1, 2, 5, 63, 1000, 4096, 4097, 50257, 151936])
def test_sample_filters(V, dtype):
    rng = np.random.default_rng(V)
    B = 5
    for i, (name, f) in enumerate(FILTERS.items()):
        x = logits_of(B, V, dtype, 7 * i + V, spread=[0.3, 2.0, 4.0][i % 3])
        if V > 8:
            x[0, 3] = 30.0                       # a confident row
        u = rng.random(B).astype(np.float32)
        u[1] = 0.0
        u[2] = 1.0 - 2.0 ** -24
        check(x, u, f"sample V {V} {dtype} {name}", temperature=[1.0, 0.7, 1.3, 0.2, 5.0],
              **{k: [v] * B for k, v in f.items()})


def test_sample_many_rows_each_with_its_own_parameters():
    rng = np.random.default_rng(5)
    for B, V, dtype in ((300, 32000, "bfloat16"), (120, 151936, "float32"), (700, 130, "float32")):
        x = logits_of(B, V, dtype, B)
        pick = lambda *a: [a[j] for j in rng.integers(0, len(a), B)]  # noqa: E731
        check(x, rng.random(B).astype(np.float32), f"sample {B} rows of {V}", temperature=pick(0.5, 1.0, 2.0, 0.0),
              top_k=pick(0, -3, 5, 200, 5000), top_p=pick(1.0, 0.5, 0.99, 2.0, float("nan")), min_p=pick(0.0, 0.1, -1.0))


def test_sample_equal_logits():
    """Ties: the lowest indices rank first, whole rows of equal logits, and
    filters that end inside a group of equal ones."""
    import torch
    for V in (8, 4000, 50000):
        x = torch.zeros(4, V, device="cuda")
        x[1] = -3.0e38
        x[2, ::2] = -1.0
        x[3] = torch.where(torch.arange(V, device="cuda") % 7 == 3, 2.0, 1.0)
        for f in (dict(), dict(top_k=3), dict(top_k=V // 2 + 1), dict(top_p=0.5), dict(top_p=0.375), dict(min_p=1.0),
                  dict(top_k=V - 2, top_p=0.25), dict(top_p=0.9999)):
            for u in (0.0, 0.3, 0.99999):
                check(x, np.full(4, u, np.float32), f"equal logits V {V} {f} u {u}", **{k: [v] * 4 for k, v in f.items()})
                check(x.to(torch.bfloat16), np.full(4, u, np.float32), "  bf16", **{k: [v] * 4 for k, v in f.items()})


def test_sample_unusable_logits_and_odd_parameters():
    import torch
    inf, nan = float("inf"), float("nan")
    V = 300
    x = logits_of(8, V, "float32", 3, holes=False)
    x[0] = -inf
    x[1] = nan
    x[2, :] = -inf
    x[2, 250] = -5.0
    x[3, 17] = nan
    x[4, 20], x[4, 200] = inf, inf
    x[5, :] = 3.0e38
    x[5, 9] = -3.0e38
    x[6, 0], x[6, 1] = -0.0, 0.0
    x[6, 2:] = -1.0e-30
    for u in (0.1, 0.6, nan, -2.0, 7.0):
        for f in (dict(), dict(top_k=2), dict(top_p=0.9), dict(min_p=0.5), dict(temperature=0.0), dict(temperature=nan),
                  dict(temperature=1e-10), dict(temperature=1e30), dict(temperature=inf), dict(temperature=-1.0),
                  dict(temperature=1e-44, top_p=0.5)):
            if u == 0.1 or "temperature" not in f:
                check(x, np.full(8, u, np.float32), f"unusable logits u {u} {f}", **{k: [v] * 8 for k, v in f.items()})


def test_sample_the_longest_row():
    V = 1 << 20
    for name in ("none", "k40", "k_many", "p", "m", "kpm"):
        x = logits_of(2, V, "bfloat16", 23, holes=False)
        check(x, np.array([0.4, 0.999], np.float32), f"sample V {V} {name}", temperature=[1.0, 3.0],
              **{k: [v] * 2 for k, v in FILTERS[name].items()})


def test_sample_the_most_rows():
    """65,536 rows, every 64th the same: the draws repeat with them."""
    import torch
    x = logits_of(64, 50, "float32", 29)
    u = torch.linspace(0, 0.99, 64, device="cuda")
    f = dict(top_k=torch.arange(64, device="cuda").int() % 7, top_p=0.4 + 0.01 * torch.arange(64, device="cuda"))
    lists = {k: v.tolist() for k, v in f.items()}
    check(x, u.cpu().numpy(), "64 of 65,536 rows", **lists)
    want = torch.tensor(draw(x, u.cpu().numpy(), **lists)[0], device="cuda")
    from paper_2608_22788_amd import binding
    token = torch.zeros(65536, dtype=torch.int32, device="cuda")
    say("65,536 rows")
    binding.sample(x.repeat(1024, 1), u.repeat(1024), token, **{k: v.repeat(1024) for k, v in f.items()})
    assert torch.equal(token.view(1024, 64), want.view(1, 64).expand(1024, 64))


def test_sample_min_p_nan_is_off():
    nan = float("nan")
    for V in (300, 20000):
        x = logits_of(4, V, "float32", 17)
        for u in (0.2, 0.99):
            check(x, np.full(4, u, np.float32), f"min-p NaN V {V} u {u}", min_p=[nan, 0.5, nan, 0.0], top_k=[0, 0, 20, 20])


def test_sample_strided_rows_and_no_log_probability():
    import torch
    from paper_2608_22788_amd import binding
    for dtype in (torch.float32, torch.bfloat16):
        full = logits_of(6, 5003, "float32", 11).to(dtype)
        x = full[:, 1:4998]
        u = np.linspace(0.05, 0.95, 6).astype(np.float32)
        want, lp = draw(x.contiguous(), u, top_p=[0.9] * 6)
        got, lq = draw(x, u, top_p=[0.9] * 6)
        assert (want == got).all() and (lp == lq).all()
        token = torch.zeros(6, dtype=torch.int32, device="cuda")
        binding.sample(x, torch.from_numpy(u).cuda(), token, top_p=torch.full((6,), 0.9, device="cuda"))
        assert (token.cpu().numpy() == want).all()


def test_sample_follows_the_distribution():
    """The draw over a uniform grid of u takes each kept token in proportion to
    its weight (to one grid point)."""
    import torch
    V, n = 40, 4000
    row = logits_of(1, V, "float32", 21, holes=False)
    u = (np.arange(n) + 0.5) / n
    f = dict(temperature=0.8, top_k=25, top_p=0.9, min_p=0.01)
    tokens, _ = draw(row.expand(n, V).contiguous(), u, **{k: [v] * n for k, v in f.items()})
    ids, w = orc.kept_tokens(row[0].cpu().numpy(), **{k: np.float32(v) if k != "top_k" else v for k, v in f.items()})
    share = np.bincount(tokens, minlength=V) / n
    expect = np.zeros(V)
    expect[ids] = w / w.sum()
    assert np.abs(share - expect).max() <= 1.0 / n + 1e-6
