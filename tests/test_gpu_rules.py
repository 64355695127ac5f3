"""GPU tests of the rules on logits against oracle/rules.py in float64.

Tolerance: up to six float32 operations (a reciprocal and a product, frequency * n, the
sum with presence, the difference, the bias) and as many additions as a token has
biases less one (at most 40 here), each off by 2^-24 of the largest magnitude met,
so 46 * 2^-24 < 2^-18 of it; a bf16 result once more by 2^-8 of itself."""
import numpy as np
import pytest

from gpu_util import say
from oracle import rules as orc

pytestmark = pytest.mark.gpu

CANARY = -77.0


def make(B, V, dtype, out_dtype=None, hist=(0, 60), biases=0, masked=False, penalties="rfp", prompt=True, seed=0,
         pad=0, in_place=False, ids=None):
    """Inputs; rows of logits and out start `pad` elements apart from their neighbours' ends."""
    import torch
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    bf = {"f": torch.float32, "b": torch.bfloat16}
    logits = torch.empty(B, V + pad, device="cuda").normal_(generator=g).mul_(4).to(bf[dtype])[:, :V]
    flat = rng.integers(0, B * V, max(1, V // 50))
    for k, odd in enumerate((float("-inf"), float("inf"), float("nan"), -0.0)):
        at = torch.from_numpy(flat[k::4]).cuda()
        logits[at // V, at % V] = odd
    out = logits if in_place else torch.full((B, V + pad + 3), CANARY, dtype=bf[out_dtype or dtype], device="cuda")[:, 2:V + 2]
    n = max(hist[1], 1)
    tokens = rng.integers(0, max(1, V // 3), (B, n + 2)) ** 2 % (V + 5) - 2 if ids is None else np.broadcast_to(ids, (B, len(ids)))
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.float32, device="cuda")  # noqa: E731
    kw = {}
    if penalties:
        lens = rng.integers(hist[0], hist[1] + 1, B)
        kw.update(tokens=i32(tokens.copy()), lens=i32(lens))
        if prompt:
            kw["prompt_lens"] = i32(rng.integers(0, lens + 1))
        rep, freq, pres = 0.5 + rng.random(B), rng.random(B) - 0.3, rng.random(B) - 0.3
        rep[B // 2], freq[B // 3], pres[B // 4] = [(0.0, np.nan, np.inf), (-1.0, np.inf, np.nan), (np.nan, 0.0, 0.0)][seed % 3]
        for c, name, v in (("r", "repetition", rep), ("f", "frequency", freq), ("p", "presence", pres)):
            if c in penalties:
                kw[name] = f32(v)
    if biases:
        count = rng.integers(0, biases + 1, B)
        count[-1] = biases
        total = int(count.sum())
        t = rng.integers(-3, V + 3, total)
        t[rng.random(total) < 0.3] = V // 2
        w = rng.normal(size=total) * 3
        w[rng.random(total) < 0.05] = -np.inf
        kw.update(bias_starts=i32(np.concatenate(([0], np.cumsum(count)))), bias_tokens=i32(t), bias_values=f32(w))
    if masked:
        words = (V + 31) // 32
        m = rng.integers(-2 ** 31, 2 ** 31, (B, words + 2))
        m[0], m[B // 2] = 0, -1
        kw["allowed"] = i32(m)[:, :words]
    return dict(logits=logits, out=out, **kw)


def check(s, tag):
    import torch
    from paper_2608_22788_amd import binding
    say(tag)
    host = {k: v.float().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for k, v in s.items()}
    before = None if s["out"] is s["logits"] else s["logits"].clone()
    rules = {k: v for k, v in s.items() if k not in ("logits", "out")}
    binding.logit_rules(s["logits"], s["out"], **rules)
    torch.cuda.synchronize()
    if before is not None:
        bits = lambda t: t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)  # noqa: E731
        assert torch.equal(bits(before), bits(s["logits"])), "logits were written"
        base = s["out"]._base
        edge = base.clone()
        edge[:, 2:2 + s["out"].shape[1]] = CANARY
        assert (edge == CANARY).all(), "written outside"
    got = s["out"].float().cpu().numpy().astype(np.float64)
    host_rules = {k: v for k, v in host.items() if k not in ("logits", "out")}
    worst = 0.0
    for b in range(got.shape[0]):
        x, size = orc.row(host["logits"][b], b, **host_rules)
        odd = ~np.isfinite(x)
        assert np.array_equal(got[b][odd], x[odd], equal_nan=True), f"{tag}: row {b}"
        err = np.abs(got[b] - np.where(odd, 0, x))[~odd]
        bar = (2.0 ** -18 * size + (2.0 ** -8 * np.abs(np.where(odd, 0, x)) if s["out"].dtype == torch.bfloat16 else 0))[~odd]
        assert (err <= bar).all(), f"{tag}: row {b}, {np.nanmax(err / bar)}"
        worst = max(worst, float((err / np.maximum(bar, 1e-30)).max()) if err.size else 0.0)
    say(f"  worst error / bound {worst:.3f}")


@pytest.mark.parametrize("types", ["ff", "bb", "bf", "fb"])
@pytest.mark.parametrize("V", [1, 7, 31, 32, 33, 1000, 8191, 8192, 8193, 20011])
def test_rules_sizes(types, V):
    for pad in (0, 3):
        check(make(5, V, types[0], types[1], biases=9, masked=True, seed=V + pad, pad=pad), f"rules {types} {V} pad {pad}")


@pytest.mark.parametrize("dtype", ["f", "b"])
@pytest.mark.parametrize("kw", [dict(), dict(penalties=""), dict(penalties="r"), dict(penalties="f", prompt=False),
                                dict(penalties="p"), dict(penalties="", biases=30), dict(penalties="", masked=True),
                                dict(biases=40), dict(masked=True), dict(biases=5, masked=True)], ids=str)
def test_rules_each(dtype, kw):
    for in_place in (False, True):
        for seed in range(3):
            check(make(4, 9001, dtype, seed=seed, in_place=in_place, **kw), f"rules {dtype} {kw} in place {in_place}")


def test_rules_vocabulary_and_long_texts():
    check(make(3, 151936, "b", hist=(30000, 50000), biases=300, masked=True, seed=1), "rules 151,936 tokens")
    check(make(2, 1 << 20, "f", hist=(0, 5), seed=2), "rules 2^20 tokens")
    check(make(200, 50257, "b", hist=(0, 3000), masked=True, seed=3, in_place=True), "rules 200 rows, odd vocabulary")
    check(make(3000, 64, "f", hist=(0, 3), seed=4), "rules 3,000 rows")


def test_rules_one_token_all_along():
    """A text of one token, of its ends' lengths, and tokens that are none."""
    for n in (1, 2, 3, 4, 5, 4095, 4096, 4097, 16385, 70001):
        check(make(2, 300, "f", hist=(n, n), seed=n, ids=np.full(n + 1, 7)), f"rules {n} times one token")
    check(make(2, 300, "f", hist=(9, 9), ids=np.array([-2 ** 31, -1, 300, 2 ** 31 - 1, 299, 0, 0, 0, 0])), "rules odd ids")


def test_rules_lengths_and_starts_out_of_range():
    import torch
    s = make(4, 500, "f", hist=(10, 20), biases=20, seed=5)
    s["lens"] = torch.tensor([-3, 10 ** 9, 5, 0], dtype=torch.int32, device="cuda")
    s["prompt_lens"] = torch.tensor([2, 10 ** 9, -5, 7], dtype=torch.int32, device="cuda")
    s["bias_starts"] = torch.tensor([-9, 10, 7, 12, 10 ** 9], dtype=torch.int32, device="cuda")
    check(s, "rules lengths out of range")


def test_rules_many_biases():
    """More than a workgroup's threads hold at once, many of one token."""
    import torch
    s = make(2, 9000, "f", penalties="", biases=1, seed=6)
    n = 5000
    t = torch.arange(n, device="cuda", dtype=torch.int32) * 7 % 9000
    t[::13] = 4
    s["bias_tokens"], s["bias_values"] = t, torch.full((n,), 0.5, device="cuda")   # (sums are exact)
    s["bias_starts"] = torch.tensor([0, 1, n], dtype=torch.int32, device="cuda")
    check(s, "rules 5,000 biases")


def test_rules_bias_sums_in_list_order():
    import torch
    from paper_2608_22788_amd import binding
    w = torch.tensor([1e8, 1.0, -1e8, 1.0, 3e7, -3e7, 0.25] * 40, device="cuda")
    order = torch.tensor([0, 280], dtype=torch.int32, device="cuda")
    x = torch.zeros(1, 5, device="cuda")
    out = torch.empty_like(x)
    binding.logit_rules(x, out, bias_starts=order, bias_tokens=torch.full((280,), 3, dtype=torch.int32, device="cuda"),
                        bias_values=w)
    want = np.float32(0)
    for v in w.cpu().numpy():
        want = np.float32(want + v)
    assert out.cpu().numpy()[0].tolist() == [0, 0, 0, float(want), 0]


def test_rules_no_text_and_empty_lists():
    import torch
    from paper_2608_22788_amd import binding
    x = torch.randn(2, 40, device="cuda")
    out = torch.empty_like(x)
    e = lambda dt: torch.empty(0, dtype=dt, device="cuda")  # noqa: E731
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    binding.logit_rules(x, out, tokens=torch.empty(2, 0, dtype=torch.int32, device="cuda"), lens=z,
                        repetition=torch.full((2,), 2.0, device="cuda"),
                        bias_starts=torch.zeros(3, dtype=torch.int32, device="cuda"), bias_tokens=e(torch.int32),
                        bias_values=e(torch.float32))
    assert torch.equal(x, out)


@pytest.mark.parametrize("types", ["ff", "bb", "bf"])
def test_rules_copies_what_no_rule_names(types):
    """Bit for bit, signed zeros and denormal values among them, with rules for
    other tokens and without any."""
    import torch
    from paper_2608_22788_amd import binding
    bf = {"f": torch.float32, "b": torch.bfloat16}
    x = torch.randn(3, 5003, device="cuda").to(bf[types[0]])
    x[:, ::7], x[:, 1::7], x[:, 2::7], x[:, 3::7] = -0.0, 0.0, -1e-39, float("-inf")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for kw in ({}, dict(bias_starts=i32([0, 1, 1, 2]), bias_tokens=i32([5002, 5002]), bias_values=torch.ones(2, device="cuda"))):
        out = torch.zeros_like(x, dtype=bf[types[1]])
        binding.logit_rules(x, out, **kw)
        want, got = x.to(bf[types[1]])[:, :5002].contiguous(), out[:, :5002].contiguous()
        bits = torch.int32 if types[1] == "f" else torch.int16
        assert torch.equal(got.view(bits), want.view(bits)), kw.keys()


def test_rules_on_more_workgroups_than_one_launch_has():
    """65,536 rows of 520,193 tokens in place (68 GB): 2^23 workgroups.  Every row
    has a bias for its last token and for one of its own; every logit is compared."""
    import torch
    from paper_2608_22788_amd import binding
    B, V = 65536, 127 * 4096 + 1
    say("rules on 65,536 rows of 520,193 tokens")
    x = torch.zeros(B, V, dtype=torch.bfloat16, device="cuda")
    row = torch.arange(B, device="cuda")
    own = row * 7919 % (V - 1)
    w = (1 + row % 7).float()
    binding.logit_rules(x, x, bias_starts=torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda"),
                        bias_tokens=torch.stack((own, torch.full_like(own, V - 1)), 1).flatten().to(torch.int32),
                        bias_values=torch.stack((w, -w), 1).flatten())
    for at, want in ((own, w), (torch.full_like(own, V - 1), -w)):
        assert torch.equal(x[row, at].float(), want)
        x[row, at] = 0.0
    for part in x.view(torch.int16).split(4096):
        assert int(part.count_nonzero()) == 0, "a token that no rule names was changed"


@pytest.mark.parametrize("dtype", ["f", "b"])
def test_rules_in_place_leave_groups_that_no_rule_names(dtype):
    """Eight neighbouring tokens without a named one keep their bits, signalling NaNs'
    too, which arithmetic would make quiet; a named token's neighbours keep their
    values."""
    import torch
    from paper_2608_22788_amd import binding
    V, kind, bits, snan = 5003, *((torch.float32, torch.int32, 0x7f800001) if dtype == "f" else
                                  (torch.bfloat16, torch.int16, 0x7f81))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.randn(3, V, device="cuda").to(kind)
    raw = x.view(bits)
    raw[:, ::5] = snan
    for text, biases in (([16, 4099], [(1, 2500), (2, 5002)]), ([0], [])):
        named = torch.zeros(3, V, dtype=torch.bool, device="cuda")
        named[:, text] = True
        for b, t in biases:
            named[b, t] = True
        group = torch.nn.functional.pad(named, (0, -V % 8)).view(3, -1, 8).any(2).repeat_interleave(8, 1)[:, :V]
        before = raw.clone()
        kw = {}
        if biases:
            kw = dict(bias_starts=i32([0, 0, 1, 2]), bias_tokens=i32([t for _, t in biases]),
                      bias_values=torch.full((2,), 3.0, device="cuda"))
        binding.logit_rules(x, x, tokens=i32([text] * 3), lens=i32([len(text)] * 3),
                            presence=torch.full((3,), 0.5, device="cuda"), **kw)
        assert torch.equal(raw[~group], before[~group])
        beside = group & ~named
        assert torch.equal(torch.nan_to_num(x[beside].float()), torch.nan_to_num(before.view(kind)[beside].float()))
        odd = before.view(kind).isnan()
        assert torch.equal(x.isnan(), odd) and (raw != before)[named & ~odd].all()


@pytest.mark.parametrize("dtype", ["f", "b"])
@pytest.mark.parametrize("V", [1, 7, 8, 9, 33, 4095, 4097, 12289])
def test_rules_in_place_sizes(dtype, V):
    for pad in (0, 3):
        check(make(5, V, dtype, biases=9, masked=True, seed=V + pad, pad=pad, in_place=True), f"rules in place {V} pad {pad}")
