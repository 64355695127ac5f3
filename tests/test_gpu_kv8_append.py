"""GPU tests of the append to the cache held in 8 bits against oracle/kv8.py.

Tolerances.  A row's value x relative to the page's power comes from float32
arithmetic that is off by 2^-18 absolute (values of at most 8, as in the bf16
append's tests), over the power; then one rounding to e4m3, half a step of the
result, where that error may move it to the next binade (a step there is twice as
large, so half a step of |x| plus its error is taken).  Powers are compared where
the largest value is not within that error of a border, everywhere for values,
which no arithmetic touches."""
import numpy as np
import pytest

from gpu_util import say
from oracle import kv8
from test_gpu_chunk import CANARY, f64, rope_inputs

pytestmark = pytest.mark.gpu


def inputs(heads, lens, rot, norm, seed=0, fused=True):
    """rope_inputs with a cache of random codes (NaN ones in unused slots) and
    powers around 2^-7."""
    import torch
    s = rope_inputs(heads, lens, rot, norm, seed=seed, fused=fused)
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    for name in ("k_pages", "v_pages"):
        unused = s[name].isnan()
        x = torch.randn(s[name].shape, generator=g, device="cuda").mul_(90).clamp_(-448, 448).to(torch.float8_e4m3fn)
        x.view(torch.uint8)[unused] = 0x7f
        s[name] = x
    n = s["k_pages"].shape[:2]
    s["scales"] = torch.randint(116, 124, (*n, 2), generator=g, device="cuda").to(torch.uint8).view(torch.float8_e8m0fnu)
    return s


def u8(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def run(s, interleaved, out, **kw):
    from paper_2608_22788_amd import binding
    binding.rope_append_kv8(s["q"], s["k"], s["v"], out, s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"],
                            s["starts"], s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6,
                            interleaved=interleaved, **kw)


def check(s, interleaved, tag, in_place=False):
    import torch
    say(tag)
    num = lambda t: None if t is None else f64(t)  # noqa: E731
    codes0, bytes0 = [u8(s["k_pages"]).copy(), u8(s["v_pages"]).copy()], u8(s["scales"]).copy()
    freq = np.zeros(0) if s["inv_freq"] is None else s["inv_freq"].cpu().numpy()
    want_q, *want, bytes1 = kv8.append(f64(s["q"]), f64(s["k"]), f64(s["v"]), *codes0, bytes0, s["table"].cpu().numpy(),
                                       s["ctx"].cpu().numpy(), s["starts"].cpu().numpy(), freq, num(s["q_norm"]),
                                       num(s["k_norm"]), 1e-6, interleaved)
    out = s["q"] if in_place else torch.full(s["q"].shape, CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    before = out.clone()
    run(s, interleaved, out)
    torch.cuda.synchronize()
    idle = np.isnan(want_q).all(axis=(1, 2))
    raw = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    assert (raw(out)[idle] == raw(before)[idle]).all(), "a row of no sequence was written"
    got, ref = f64(out)[~idle], want_q[~idle]
    fine = np.isfinite(ref)
    assert (np.isfinite(got) == fine).all()
    assert (np.abs(got - ref)[fine] <= (2.0 ** -8 * np.abs(ref) + 2.0 ** -18)[fine]).all(), f"{tag}: queries"
    got_bytes = u8(s["scales"])
    for which in (0, 1):
        codes = u8(s["k_pages"] if which == 0 else s["v_pages"])
        w = want[which]
        alone = np.isnan(w)
        assert (codes[alone] == codes0[which][alone]).all(), f"{tag}: a slot that nothing goes to was written"
        moved = got_bytes[..., which] != bytes1[..., which]
        if moved.any():   # a border: the other power, by one, and a largest value next to it
            assert which == 0, f"{tag}: powers of values"
            most = np.nanmax(np.where(np.isfinite(w), np.abs(w), 0), axis=(2, 3))[moved] * np.exp2(bytes1[moved][:, 0] - 127.0)
            m, e = np.frexp(most)
            assert (np.abs(m - 0.875) * np.exp2(e) <= 2.0 ** -18).all(), f"{tag}: powers of keys"
        shift = np.exp2(bytes1[..., which].astype(float) - got_bytes[..., which])[..., None, None]
        x = w * shift
        power = np.exp2(got_bytes[..., which] - 127.0)[..., None, None]
        v = kv8.code_values()[codes]
        nan = np.isinf(x)
        assert (np.isnan(v) == nan)[~alone].all(), f"{tag}: NaN codes"
        sure = ~alone & ~nan
        slack = np.broadcast_to(2.0 ** -18 / power if which == 0 else 0.0, x.shape)[sure]
        err, bar = np.abs(v[sure] - x[sure]), kv8.half_step(np.abs(x[sure]) + slack) + slack
        say(f"  {'keys' if which == 0 else 'values'}: {sure.sum()} codes, worst error / bound {(err / bar).max() if err.size else 0:.4f}")
        assert (err <= bar).all(), tag


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (5, 1, 128), (64, 4, 128), (3, 3, 64)], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["none", "both", "q", "k"])
def test_append(heads, interleaved, norm):
    D = heads[2]
    for rot in (D, D // 2, 16, 0):
        s = inputs(heads, ([1, 0, 37, 2, 16, 17], [0, 5, 15, 2000, 32, 31]), rot, norm, seed=rot)
        check(s, interleaved, f"append {heads} rot {rot} {interleaved} {norm}", in_place=rot == D // 2)


@pytest.mark.parametrize("past", range(0, 18, 1))
def test_append_every_place_in_a_page(past):
    s = inputs((4, 2, 64), ([1, 2, 15, 16, 33], [past] * 5), 64, "none", seed=past)
    check(s, False, f"append behind {past}", in_place=True)


def test_append_many_sequences():
    rng = np.random.default_rng(1)
    q = rng.integers(0, 4, 300).tolist()
    check(inputs((4, 2, 64), (q, rng.integers(0, 90, 300).tolist()), 64, "k", seed=2), False, "append 300 sequences")
    check(inputs((2, 1, 128), ([1] * 4096, rng.integers(0, 17, 4096).tolist()), 128, "none", seed=3), False,
          "append 4096 sequences")


def test_append_raises_and_keeps_powers():
    """Tokens one by one: the page's power follows its largest value so far, and
    what is held keeps its value to one rounding until it is denormal."""
    import torch
    s = inputs((2, 1, 64), ([1], [0]), 0, "none", seed=5)
    full = [2.0 ** -20, 2.0 ** -20, 3.0, 2.9, 100.0, 2.0 ** -3, 0.0, 500.0, 4.0 ** 20, 1.0, 1e-30, 7.0, 2.0 ** 21, 1, 2, 3]
    s["table"] = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    for i, size in enumerate(full):
        s["k"].normal_().clamp_(-1, 1).mul_(size)
        s["v"].normal_().clamp_(-1, 1).mul_(size)
        s["ctx"] = torch.tensor([i + 1], dtype=torch.int32, device="cuda")
        check(s, False, f"append token {i} of size {size}")


def test_append_odd_values():
    import torch
    s = inputs((4, 2, 128), ([20, 3], [10, 40]), 128, "none", seed=6)
    inf, nan = float("inf"), float("nan")
    s["v"][0, 0, 5], s["v"][3, 1, 7], s["v"][4, 0, 9], s["v"][8] = inf, -inf, nan, nan
    s["v"][21] = 3e38                      # larger than what the largest power holds
    s["v"][22] = 0.0
    check(s, False, "append odd values")
    s = inputs((4, 2, 128), ([20, 3], [10, 40]), 0, "none", seed=7)
    s["k"][2, 0, 3], s["k"][5, 1], s["k"][21] = inf, nan, -3e38
    s["v"].zero_()
    check(s, False, "append odd keys")


def test_append_skips_rows_outside_the_pool():
    import torch
    s = inputs((8, 2, 64), ([3, 3, 3], [20, 20, 20]), 64, "none", seed=4)
    s["table"][0, 1] = -1                       # a page id below the pool
    s["table"][1, 1] = s["k_pages"].shape[0]    # and above it
    s["ctx"][2] = 1                             # two rows in front of position 0
    check(s, False, "append outside the pool")
    s["starts"] = torch.tensor([0, 3, 6, 2000000], dtype=torch.int32, device="cuda")
    s["ctx"][2] = 23
    check(s, False, "append starts past the rows")
    s["starts"] = torch.tensor([0, 0, 11, 11], dtype=torch.int32, device="cuda")
    s["ctx"] = torch.tensor([5, 0, 7], dtype=torch.int32, device="cuda")
    check(s, False, "append a sequence without a length")


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_frequencies_at_any_element(interleaved):
    """Frequencies that start at no multiple of 16 bytes, and end with their memory's last."""
    import torch
    for heads in ((12, 1, 128), (4, 2, 64)):
        s = inputs(heads, ([1, 20, 40], [7, 0, 1000]), 48, "both", seed=9)
        for offset in (1, 2, 3):
            freq = torch.full((s["inv_freq"].numel() + offset,), float("nan"), device="cuda")
            freq[offset:] = s["inv_freq"]
            t = dict(s, inv_freq=freq[offset:])
            check(t, interleaved, f"append {heads} frequencies {offset} elements on {interleaved}")


def test_append_again_changes_nothing():
    """A second call with the same rows writes the same bytes: what it raised is raised."""
    import torch
    s = inputs((8, 2, 128), ([1, 5, 40], [3, 30, 100]), 128, "k", seed=8)
    out = torch.empty_like(s["q"])
    run(s, False, out)
    first = [u8(s[n]).copy() for n in ("k_pages", "v_pages", "scales")]
    run(s, False, out)
    for a, n in zip(first, ("k_pages", "v_pages", "scales")):
        assert (a == u8(s[n])).all(), n


@pytest.mark.parametrize("rejected", [1, 3])
def test_append_behind_rejected_drafts(rejected):
    """A draft block whose last row is large, of which the last `rejected` rows are taken
    back, and rows in their place: the page keeps the power that they raised, and the
    accepted tokens one rounding more, until it is filled from its first slot on."""
    import torch
    first = inputs((4, 2, 64), ([6], [0]), 0, "none", seed=10)
    cache = {n: first[n] for n in ("k_pages", "v_pages", "scales", "table")}
    said = {"k": [], "v": []}

    def step(tokens, past, tag, big=None):
        s = dict(inputs((4, 2, 64), ([tokens], [past]), 0, "none", seed=11 + past), **cache)
        if big is not None:
            for n in said:
                s[n][tokens - 1] *= big            # (rows behind belong to no sequence)
        check(s, False, tag)
        for n in said:
            said[n] = said[n][:past] + list(f64(s[n])[:tokens])

    step(6, 0, "accepted tokens")
    step(4, 6, "a draft block", big=2.0 ** 12)
    raised = u8(cache["scales"])[int(cache["table"][0, 0])].copy()
    step(3, 10 - rejected, "behind rejected drafts")
    pid = int(cache["table"][0, 0])
    assert (u8(cache["scales"])[pid] == raised).all(), "the page's power after drafts were taken back"
    for which, (n, pages) in enumerate((("k", "k_pages"), ("v", "v_pages"))):
        power = np.exp2(raised[:, which] - 127.0)[:, None, None]
        held = kv8.code_values()[u8(cache[pages])[pid]] * power
        x = np.stack(said[n], 1)                                   # [heads][tokens][D], exact (no norm, no rotation)
        err = np.abs(held[:, :x.shape[1]] - x)
        assert (err <= 2.0 ** -4 * np.abs(x) + 2 * 2.0 ** -10 * power).all(), f"{n}: two roundings"
    step(2, 0, "the page from its first slot on")
    assert (u8(cache["scales"])[pid] < raised).all()
