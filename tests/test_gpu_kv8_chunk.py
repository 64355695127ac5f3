"""GPU tests of chunk attention over the cache held in 8 bits, every output
element against oracle/chunk.py on the values that the codes stand for, with the
tolerances of test_gpu_chunk.py (cached values are exact in bf16)."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_chunk import CANARY, SHAPES, f64, make
from test_gpu_kv8_decode import NAN, eight_bits, largest_power, reference8, within

pytestmark = pytest.mark.gpu


def make8(heads, q_lens, past, seed=0, **kw):
    return eight_bits(make(*heads, q_lens, past, seed=seed, **kw), seed)


def reference(s):
    return reference8(s, f64(s["q"]), s["starts"].cpu().numpy())


def run(s, out=None, **kw):
    import torch
    from paper_2608_22788_amd import binding
    if out is None:
        T, Hq, D = s["q"].shape
        full = torch.full((T + 2, Hq + 1, D), CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        out = full[1:T + 1, :Hq]
    binding.chunk_attn_kv8(s["q"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["starts"], out,
                           s["scale"], max_q_len=s["max_q"], max_ctx_len=s["max_ctx"], **kw)
    torch.cuda.synchronize()
    return out


def check(s, tag, ref=None, **kw):
    import torch
    say(tag, kw)
    out = run(s, **kw)
    raw, got, (want, mag) = out._base.view(torch.int16), f64(out), ref or reference(s)
    rows = np.isnan(want).all(axis=(1, 2)) & np.isnan(mag).all(axis=(1, 2))   # rows of no sequence
    assert (raw[0] == CANARY).all() and (raw[-1] == CANARY).all() and (raw[:, -1] == CANARY).all(), "written outside"
    assert (raw[1:-1, :-1].cpu().numpy()[rows] == CANARY).all(), "a row of no sequence was written"
    within(got[~rows], want[~rows], mag[~rows], tag)


@pytest.mark.parametrize("heads", SHAPES, ids=str)
@pytest.mark.parametrize("lens", [
    ([1], [0]), ([1], [700]), ([17], [0]), ([64], [64]), ([129], [63]),
    ([1, 0, 33, 5, 0], [100, 50, 0, 16, 0]), ([130, 1, 1, 70], [1, 15, 16, 300])], ids=str)
def test_small(heads, lens):
    s = make8(heads, *lens, seed=3, tail_rows=2)
    ref = reference(s)
    for workers in (0, 1, 7):
        check(s, f"chunk8 {heads} {lens}", ref, num_workers=workers)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (3, 1, 128)], ids=str)
@pytest.mark.parametrize("past", [0, 1, 15, 16, 63, 64, 65, 127, 128, 129, 191, 192, 255, 256, 320])
def test_every_number_of_tiles(heads, past):
    """One to six KV tiles of a row tile: the places that codes and tiles take in LDS."""
    s = make8(heads, [1, 3, 66], [past, max(past - 2, 0), past], seed=past)
    ref = reference(s)
    for workers in (0, 1, 2):
        check(s, f"chunk8 {heads} past {past}", ref, num_workers=workers)


@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 4, 128), (8, 2, 64)], ids=str)
def test_long(heads):
    s = make8(heads, [300, 1, 700, 2], [1000, 3000, 0, 4097], seed=5)
    ref = reference(s)
    for workers in (0, 3, 100, 999):
        check(s, f"chunk8 long {heads}", ref, num_workers=workers)


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64)], ids=str)
def test_values_that_a_row_does_not_see(heads):
    """NaN codes of keys and values behind a row's own position, and in front of it."""
    s = make8(heads, [70, 20, 200], [30, 0, 130], seed=8)
    tab = s["table"].cpu().numpy()
    import torch

    def plant(name, b, t, g, d):
        s[name].view(torch.uint8)[int(tab[b, t // 16]), g, t % 16, d] = NAN

    plant("v_pages", 0, 95, 0, 3)        # seen by the last rows only
    plant("v_pages", 0, 60, 1, 50)
    plant("v_pages", 1, 19, 0, slice(0, heads[2]))
    plant("k_pages", 1, 18, 1, 5)        # the last two rows' scores
    plant("v_pages", 2, 10, 0, 63)       # seen by every row
    plant("v_pages", 2, 290, 1, 31)
    ref = reference(s)
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
    for workers in (0, 1, 5, 64):
        check(s, "chunk8 odd values", ref, num_workers=workers)


def test_rows_in_front_of_position_zero_and_bad_pages():
    import torch
    for D in (64, 128):
        s = make8((8, 2, D), [40, 10, 90, 5, 2], [0, 0, 100, 60, 900], seed=9)
        s["ctx"] = torch.tensor([25, 0, 190, 65, 902], dtype=torch.int32, device="cuda")   # fewer keys than rows
        s["table"][2, 3] = -1
        s["table"][3, 1] = s["k_pages"].shape[0]
        s["table"][3, 2] = 2 ** 31 - 1
        s["table"][4, 5:40:3] = -9          # in every wavefront's pages, tile after tile
        ref = reference(s)
        for workers in (0, 1, 9):
            check(s, "chunk8 rows without keys, bad pages", ref, num_workers=workers)
        s["starts"] = torch.tensor([-5, 40, 50, 140, 145, 9000], dtype=torch.int32, device="cuda")
        check(s, "chunk8 starts past the rows")


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_scales(scale):
    s = make8((8, 2, 128), [70, 3], [30, 500], seed=10)
    s["scale"] = scale
    s["q"].mul_(0.25)
    check(s, f"chunk8 scale {scale}")


def test_powers_of_any_size():
    import torch
    s = make8((32, 8, 128), [100, 1], [300, 70], seed=4)
    g = torch.Generator(device="cuda").manual_seed(1)
    b = s["scales"].view(torch.uint8)
    b[..., 0] = torch.randint(100, 120, b.shape[:2], generator=g, device="cuda").to(torch.uint8)
    b[..., 1] = torch.randint(27, 228, b.shape[:2], generator=g, device="cuda").to(torch.uint8)
    check(s, "chunk8 powers")


def test_in_place_and_workspace_contents():
    import torch
    from paper_2608_22788_amd import binding
    s = make8((8, 2, 128), [100, 1, 30], [1000, 700, 0], seed=13)
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])
    ws = torch.full((binding.chunk_kv8_workspace_size(shape),), 255, dtype=torch.uint8, device="cuda")
    a = run(s).clone()
    assert torch.equal(a, run(s, workspace=ws))
    run(s, out=s["q"])
    assert torch.equal(a, s["q"])


def test_many_sequences_and_pieces():
    rng = np.random.default_rng(2)
    q = rng.integers(0, 4, 300).tolist()
    s = make8((4, 2, 64), q, rng.integers(0, 90, 300).tolist(), seed=20)
    check(s, "chunk8 300 sequences")
    check(s, "chunk8 300 sequences", num_workers=777)
    s = make8((2, 1, 64), [3], [40000], seed=21)
    ref = reference(s)
    for workers in (0, 500, 1300):
        check(s, "chunk8 one unit in many pieces", ref, num_workers=workers)
    for D in (64, 128):
        check(make8((2, 1, D), [1] * 4096, [0] * 4096, seed=22), f"chunk8 4096 sequences, head_dim {D}")


@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 1, 128), (8, 2, 64), (5, 5, 64)], ids=str)
def test_few_rows_behind_long_contexts(heads):
    """Row tiles of up to 16 rows, whose wavefronts share the keys, beside larger
    ones: more pages than a wavefront keeps the ids of, and each end of a page."""
    few = max(16 * heads[1] // heads[0], 1)
    s = make8(heads, [1, few, few + 1, 1, 2, 300, 1], [20000, 8191, 8192, 8193, 32, 40, 0], seed=31)
    ref = reference(s)
    for workers in (0, 1, 2, 7, 300):
        check(s, f"chunk8 few rows {heads}", ref, num_workers=workers)


@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_odd_values_and_pages(D):
    """NaN codes that one of a few rows sees, bad pages, rows in front of position zero."""
    import torch
    s = make8((8, 2, D), [4, 2, 3, 4], [700, 29, 9000, 0], seed=32)
    tab = s["table"].cpu().numpy()

    def plant(name, b, t, g, d):
        s[name].view(torch.uint8)[int(tab[b, t // 16]), g, t % 16, d] = NAN

    plant("v_pages", 0, 703, 0, 3)       # the last row's own
    plant("v_pages", 0, 701, 1, slice(0, D))
    plant("k_pages", 0, 702, 1, 9)
    plant("v_pages", 1, 30, 0, 5)
    plant("v_pages", 2, 40, 1, D - 1)    # seen by every row
    s["table"][2, 100:500:7] = -1
    s["table"][2, 3] = s["k_pages"].shape[0]
    s["ctx"][3] = 2                      # two rows have no key
    ref = reference(s)
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
    for workers in (0, 1, 3, 50):
        check(s, f"chunk8 few rows, odd values {D}", ref, num_workers=workers)


def test_pages_behind_4_gib():
    import torch
    s = make8((32, 8, 128), [20, 1], [150, 40], seed=8)
    ref = reference(s)
    table, n, pages = s["table"].long(), s["k_pages"].shape[0], 300001
    place = torch.randperm(pages - 262200, device="cuda")[:n] + 262200     # behind 4 GiB
    place[0] = pages - 1
    place = place.unique()
    place = torch.cat((place, torch.arange(262200 - n, 262200 - place.numel(), device="cuda")))[:n]
    for name, dt in (("k_pages", torch.float8_e4m3fn), ("v_pages", torch.float8_e4m3fn), ("scales", torch.float8_e8m0fnu)):
        far = torch.empty(pages, *s[name].shape[1:], dtype=dt, device="cuda")
        far.view(torch.uint8)[place] = s[name].view(torch.uint8)
        s[name] = far
    s["table"] = torch.where(table >= 0, place[table.clamp(min=0)], table).to(torch.int32).contiguous()
    check(s, "chunk8 far pages", ref)


@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 1, 128), (8, 2, 64)], ids=str)
def test_the_largest_power(heads):
    """As in test_gpu_kv8_decode.py: in row tiles of few rows and of many."""
    q = [1, 5, 70, 3]
    s = make8(heads, q, [99, 700, 26, 0], seed=12)
    largest_power(s, [n - min(k, 3) + 1 for n, k in zip(s["ctx"].tolist(), q)])   # the last one or two rows see some
    want, mag = reference(s)
    ends = np.cumsum(q)
    keep = np.ones(int(ends[-1]), dtype=bool)
    for e, n in zip(ends, q):
        keep[e - min(n, 3) + 1:e] = False
    for workers in (0, 1, 5, 64):
        say("chunk8 largest power", heads, workers)
        within(f64(run(s, num_workers=workers))[keep], want[keep], mag[keep], f"chunk8 largest power {heads}")
