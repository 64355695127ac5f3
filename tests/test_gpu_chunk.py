"""GPU tests of the operators on packed rows: chunk attention and rotation with
append, against oracle/chunk.py in float64.

Tolerances of chunk attention, per element: probabilities are rounded to bf16
before the value product (relative 2^-8 each, so at most 2^-8 sum p |v|), the
result once more (2^-8 of it), and scores carry float32 rounding: a dot
product of D = 128 terms is off by at most D 2^-24 sum |q k| < 2^-17 x 128,
times the scale 2^-3.5, i.e. 2^-13.5 on the exponent for the N(0, 1) inputs here,
and the exponential by 2^-22; 2^-10 covers both.  So
    |out - ref| <= 2^-8 (|ref| + A) + 2^-10 A,  A = sum p |v|.
"""
import numpy as np
import pytest

from oracle import chunk as orc
from gpu_util import say

pytestmark = pytest.mark.gpu


def make(Hq, Hkv, D, q_lens, past, seed=0, spare=3, tail_rows=0, fused=True, poison=True):
    """Packed inputs on the GPU, and their values as float64 numpy arrays.  Every
    slot that no token fills, and the spare pages, hold NaN."""
    import torch
    rng = np.random.default_rng(seed)
    ctx = [int(q + p) for q, p in zip(q_lens, past)]
    B, T = len(q_lens), int(sum(q_lens)) + tail_rows
    npg = [(n + 15) // 16 for n in ctx]
    total = sum(npg) + spare
    perm = rng.permutation(total).astype(np.int32)
    table = np.full((B, max(max(npg), 1) + 2), -7, dtype=np.int32)      # entries past the context are not ids
    at = 0
    for b, n in enumerate(npg):
        table[b, :n] = perm[at:at + n]
        at += n
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    normal = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    kp, vp = normal(total, Hkv, 16, D), normal(total, Hkv, 16, D)
    if poison:
        used = np.zeros((total, 16), dtype=bool)
        for b, n in enumerate(ctx):
            for j in range(npg[b]):
                used[table[b, j], :min(16, n - 16 * j)] = True
        mask = torch.from_numpy(~used).cuda()[:, None, :, None]
        kp.masked_fill_(mask, float("nan"))
        vp.masked_fill_(mask, float("nan"))
    qkv = normal(max(T, 1), Hq + 2 * Hkv, D)[:T]
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    starts = np.concatenate(([0], np.cumsum(q_lens)))
    return dict(q=q, k=k, v=v, k_pages=kp, v_pages=vp, table=i32(table), ctx=i32(ctx), starts=i32(starts),
                scale=D ** -0.5, max_q=int(max(q_lens)), max_ctx=max(max(ctx), 1))


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def reference(s):
    return orc.chunk_attention(f64(s["q"]), f64(s["k_pages"]), f64(s["v_pages"]), s["table"].cpu().numpy(),
                               s["ctx"].cpu().numpy(), s["starts"].cpu().numpy(), s["scale"])


CANARY = 0x5A5A


def run_chunk(s, num_workers=0, out=None, **kw):
    import torch
    from paper_2608_22788_amd import binding
    if out is None:
        T, Hq, D = s["q"].shape
        full = torch.full((T + 2, Hq + 1, D), CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        out = full[1:T + 1, :Hq]
    binding.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], out, s["scale"],
                       max_q_len=s["max_q"], max_ctx_len=s["max_ctx"], num_workers=num_workers, **kw)
    torch.cuda.synchronize()
    return out


def check_chunk(s, tag, num_workers=0, ref=None):
    import torch
    say(tag, "workers", num_workers)
    out = run_chunk(s, num_workers)
    full = out._base
    got, (want, mag) = f64(out), ref or reference(s)
    raw = full.view(torch.int16)
    rows = np.isnan(want).all(axis=(1, 2)) & np.isnan(mag).all(axis=(1, 2))   # rows of no sequence
    assert (raw[0] == CANARY).all() and (raw[-1] == CANARY).all() and (raw[:, -1] == CANARY).all(), "written outside"
    assert (raw[1:-1, :-1].cpu().numpy()[rows] == CANARY).all(), "a row of no sequence was written"
    g, w, m = got[~rows], want[~rows], mag[~rows]
    assert (np.isnan(g) == np.isnan(w)).all(), f"{tag}: NaN where there is none, or none where there is one"
    inf = np.isinf(w)
    assert (g[inf] == w[inf]).all(), f"{tag}: infinities differ"
    fine = np.isfinite(w)
    err = np.abs(g - w)[fine]
    bar = (2.0 ** -8 * (np.abs(w) + m) + 2.0 ** -10 * m)[fine]
    worst = float((err / np.maximum(bar, 1e-30)).max()) if err.size else 0.0
    say(f"  worst error / bound {worst:.3f}, max {err.max() if err.size else 0:.2e}")
    assert worst <= 1.0, tag


SHAPES = [(32, 8, 128), (8, 2, 64), (4, 4, 128), (16, 1, 128), (6, 2, 64), (10, 2, 128), (7, 1, 64)]


@pytest.mark.parametrize("heads", SHAPES, ids=str)
@pytest.mark.parametrize("lens", [
    ([1], [0]), ([1], [700]), ([17], [0]), ([64], [64]), ([129], [63]),
    ([1, 0, 33, 5, 0], [100, 50, 0, 16, 0]), ([130, 1, 1, 70], [1, 15, 16, 300])], ids=str)
def test_chunk_small(heads, lens):
    s = make(*heads, *lens, seed=3, tail_rows=2)
    ref = reference(s)
    for workers in (0, 1, 7):
        check_chunk(s, f"chunk {heads} {lens}", workers, ref)


@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 4, 128), (8, 2, 64)], ids=str)
def test_chunk_long(heads):
    s = make(*heads, [300, 1, 700, 2], [1000, 3000, 0, 4097], seed=5)
    ref = reference(s)
    for workers in (0, 3, 100, 999):
        check_chunk(s, f"chunk long {heads}", workers, ref)


# ---- rotation and append ----------------------------------------------------------

def rope_inputs(heads, lens, rot, norm, seed=0, fused=True, far=0):
    import torch
    q_lens, past = lens
    s = make(*heads, q_lens, past, seed=seed, tail_rows=2, fused=fused)
    g = torch.Generator(device="cuda").manual_seed(seed + 9)
    D = heads[2]
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, device="cuda").double() / max(rot, 1))).float() if rot else None
    weight = lambda: (1.0 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)  # noqa: E731
    s["q_norm"] = weight() if norm in ("both", "q") else None
    s["k_norm"] = weight() if norm in ("both", "k") else None
    return s


def check_rope(s, interleaved, tag, in_place=False):
    """float32 arithmetic of a few operations and an angle good to 2^-23 turn on
    values of at most 8 (norm weights included): 2^-18 absolute; the rounding to
    bf16: 2^-8 relative."""
    import torch
    from paper_2608_22788_amd import binding
    say(tag)
    num = lambda t: None if t is None else f64(t)  # noqa: E731
    kp0, vp0 = s["k_pages"].clone(), s["v_pages"].clone()
    freq = np.zeros(0) if s["inv_freq"] is None else s["inv_freq"].cpu().numpy()
    want = orc.rope_append(f64(s["q"]), f64(s["k"]), f64(s["v"]), f64(kp0), f64(vp0), s["table"].cpu().numpy(),
                           s["ctx"].cpu().numpy(), s["starts"].cpu().numpy(), freq, num(s["q_norm"]),
                           num(s["k_norm"]), 1e-6, interleaved)
    q0 = s["q"].clone()
    out = s["q"] if in_place else torch.full(s["q"].shape, CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    before = out.clone()
    binding.rope_append(s["q"], s["k"], s["v"], out, s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"],
                        s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6, interleaved=interleaved)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(s["q"].view(torch.int16), q0.view(torch.int16))
    idle = np.isnan(want[0]).all(axis=(1, 2))
    raw = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    assert (raw(out)[idle] == raw(before)[idle]).all(), "a row of no sequence was written"
    for got, ref, old in ((out, want[0], None), (s["k_pages"], want[1], kp0), (s["v_pages"], want[2], vp0)):
        g = f64(got)
        if old is None:
            g, ref = g[~idle], ref[~idle]
        same = np.isnan(ref)
        assert (np.isnan(g) == same).all()
        err, bar = np.abs(g - ref)[~same], (2.0 ** -8 * np.abs(ref) + 2.0 ** -18)[~same]
        assert (err <= bar).all(), f"{tag}: {(err / bar).max()}"
    # what no row writes keeps its bits (and values are copied bit for bit)
    untouched = (s["v_pages"].view(torch.int16) == vp0.view(torch.int16)).all(-1)
    moved = s["k_pages"].view(torch.int16)[untouched] != kp0.view(torch.int16)[untouched]
    assert not bool(moved.any())


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (5, 1, 128), (64, 4, 128), (3, 3, 64)], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["none", "both", "q", "k"])
def test_rope_append(heads, interleaved, norm):
    D = heads[2]
    for rot in (D, D // 2, 16, 0):
        s = rope_inputs(heads, ([1, 0, 37, 2], [0, 5, 15, 2000]), rot, norm, seed=rot)
        check_rope(s, interleaved, f"rope {heads} rot {rot} {interleaved} {norm}", in_place=rot == D // 2)


def test_rope_far_positions_and_many_sequences():
    import torch
    s = rope_inputs((8, 2, 64), ([1] * 150, [0] * 150), 64, "none", seed=4)
    # positions near 2^24 through a page table that repeats its pages
    rng = np.random.default_rng(1)
    far = rng.integers(1 << 20, 1 << 24, 150).astype(np.int32)
    table = np.zeros((150, (1 << 20) + 1), dtype=np.int32)
    table[np.arange(150), (far - 1) // 16] = np.arange(150)
    s["table"], s["ctx"] = torch.from_numpy(table).cuda(), torch.from_numpy(far).cuda()
    check_rope(s, False, "rope far positions")


def test_rope_skips_rows_outside_the_pool():
    import torch
    s = rope_inputs((8, 2, 64), ([3, 3, 3], [20, 20, 20]), 64, "none", seed=4)
    s["table"][0, 1] = -1                       # a page id below the pool
    s["table"][1, 1] = s["k_pages"].shape[0]    # and above it
    s["ctx"][2] = 1                             # two rows in front of position 0
    check_rope(s, False, "rope outside the pool")
    s["starts"] = torch.tensor([0, 3, 6, 2000000], dtype=torch.int32, device="cuda")
    s["ctx"][2] = 23
    check_rope(s, False, "rope starts past the rows")


def test_chunk_values_that_a_row_does_not_see():
    """Infinite and NaN keys and values behind a row's own position, and infinite
    values in front of it."""
    import torch
    s = make(8, 2, 128, [70, 20, 200], [30, 0, 130], seed=8)
    tab = s["table"].cpu().numpy()

    def plant(pages, b, t, g, d, x):
        pages[int(tab[b, t // 16]), g, t % 16, d] = x

    inf, nan = float("inf"), float("nan")
    plant(s["v_pages"], 0, 95, 0, 3, nan)       # seen by the last rows only
    plant(s["v_pages"], 0, 60, 1, 100, inf)
    plant(s["v_pages"], 0, 61, 1, 100, -inf)    # rows that see both: NaN
    plant(s["v_pages"], 0, 80, 1, 17, -inf)
    plant(s["v_pages"], 1, 19, 0, slice(0, 128), nan)
    plant(s["k_pages"], 1, 18, 1, 5, nan)       # the last two rows' scores
    plant(s["v_pages"], 2, 10, 0, 64, inf)      # seen by every row
    plant(s["v_pages"], 2, 290, 1, 31, inf)
    ref = reference(s)
    assert np.isnan(ref[0]).sum() and np.isposinf(ref[0]).sum() and np.isneginf(ref[0]).sum()
    for workers in (0, 1, 5, 64):
        check_chunk(s, "chunk odd values", workers, ref)


def test_chunk_rows_in_front_of_position_zero_and_bad_pages():
    import torch
    s = make(8, 2, 64, [40, 10, 90, 5], [0, 0, 100, 60], seed=9)
    s["ctx"] = torch.tensor([25, 0, 190, 65], dtype=torch.int32, device="cuda")   # fewer keys than rows
    s["table"][2, 3] = -1
    s["table"][3, 1] = s["k_pages"].shape[0]
    s["table"][3, 2] = 2 ** 31 - 1
    ref = reference(s)
    for workers in (0, 1, 9):
        check_chunk(s, "chunk rows without keys, bad pages", workers, ref)
    s["starts"] = torch.tensor([-5, 40, 50, 140, 9000], dtype=torch.int32, device="cuda")
    check_chunk(s, "chunk starts past the rows", 4)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_chunk_scales(scale):
    s = make(8, 2, 128, [70, 3], [30, 500], seed=10)
    s["scale"] = scale
    s["q"].mul_(0.25)     # |scale * score| stays below 2^8, where float32 scores are good to 2^-13
    check_chunk(s, f"chunk scale {scale}")


def test_chunk_large_scores():
    """Rows whose largest score lies far above the others', and keys in rising
    order, which raise the running maximum tile by tile."""
    s = make(4, 2, 64, [80], [400], seed=12, poison=False)
    tab = s["table"].cpu().numpy()
    s["q"].fill_(0.5)
    for t in range(480):
        s["k_pages"][int(tab[0, t // 16]), :, t % 16] = t * 2.0 ** -3     # scores 0.25 t (exact in bf16 to 2^-1)
    check_chunk(s, "chunk rising scores")


def test_chunk_workspace_contents_do_not_matter():
    import torch
    s = make(8, 2, 128, [100, 1, 30], [1000, 700, 0], seed=13)
    from paper_2608_22788_amd import binding
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])
    ws = torch.full((binding.chunk_workspace_size(shape),), 255, dtype=torch.uint8, device="cuda")
    a = run_chunk(s).clone()
    b = run_chunk(s, workspace=ws).clone()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_chunk_many_sequences_and_pieces():
    """More sequences than one wavefront's lanes, empty ones among them; more
    pieces of a unit than the merge holds at once; as many sequences as a call
    takes."""
    rng = np.random.default_rng(2)
    q = rng.integers(0, 4, 300).tolist()
    s = make(4, 2, 64, q, rng.integers(0, 90, 300).tolist(), seed=20)
    check_chunk(s, "chunk 300 sequences", 0)
    check_chunk(s, "chunk 300 sequences", 777)
    s = make(2, 1, 64, [3], [40000], seed=21)
    ref = reference(s)
    for workers in (0, 500, 1300):
        check_chunk(s, "chunk one unit in many pieces", workers, ref)
    for D in (64, 128):
        s = make(2, 1, D, [1] * 4096, [0] * 4096, seed=22)
        check_chunk(s, f"chunk 4096 sequences, head_dim {D}", 0)
