"""GPU tests of decode and verify attention over the cache held in 8 bits, every
output element against oracle/chunk.py on the values that the codes stand for.

Tolerances are those of chunk attention (test_gpu_chunk.py): cached values are
exact in bf16, weights are rounded to it (2^-8 each), the result once more, scores
carry float32 rounding (2^-10 covers it):
    |out - ref| <= 2^-8 (|ref| + A) + 2^-10 A,  A = sum p |v|."""
import numpy as np
import pytest

from gpu_util import say
from oracle import chunk as orc
from oracle import kv8
from test_gpu_chunk import CANARY, f64, make
from test_gpu_group import CASES, SPARSE

pytestmark = pytest.mark.gpu

NAN = 0x7f


def eight_bits(s, seed=0, lo=118, hi=122):
    """The cache of `s` replaced by random codes with powers 2^(lo - 127) .. 2^(hi - 128);
    NaN codes in slots that no token fills."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    for name in ("k_pages", "v_pages"):
        unused = s[name].isnan()
        x = torch.randn(s[name].shape, generator=g, device="cuda").mul_(90).clamp_(-448, 448).to(torch.float8_e4m3fn)
        x.view(torch.uint8)[unused] = NAN
        s[name] = x
    n = s["k_pages"].shape[:2]
    s["scales"] = torch.randint(lo, hi, (*n, 2), generator=g, device="cuda").to(torch.uint8).view(torch.float8_e8m0fnu)
    return s


def make8(heads, q_lens, ctx, seed=0, qmax=None):
    """Decode inputs: q [B][Qmax][Hq][D], lengths that count the new tokens."""
    import torch
    past = [n - q for n, q in zip(ctx, q_lens)]
    s = eight_bits(make(*heads, q_lens, past, seed=seed), seed)
    B, qmax = len(q_lens), qmax or max(max(q_lens), 1)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    s["q4"] = torch.empty(B, qmax, heads[0], heads[2], dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    s["ql"] = torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    return s


def reference8(s, q, starts):
    table, scales = s["table"].cpu().numpy(), s["scales"].view(__import__("torch").uint8).cpu().numpy()
    u8 = lambda t: t.view(__import__("torch").uint8).cpu().numpy()  # noqa: E731
    return orc.chunk_attention(q, kv8.values(u8(s["k_pages"]), scales, 0), kv8.values(u8(s["v_pages"]), scales, 1), table,
                               s["ctx"].cpu().numpy(), starts, s["scale"])


def decode_reference(s):
    q, ql = f64(s["q4"]), s["ql"].cpu().numpy()
    packed = np.concatenate([q[b, :n] for b, n in enumerate(ql)])
    return reference8(s, packed, np.concatenate(([0], np.cumsum(ql))))


def within(got, want, mag, tag):
    assert (np.isnan(got) == np.isnan(want)).all(), f"{tag}: NaN where there is none, or none where there is one"
    fine = np.isfinite(want)
    err, bar = np.abs(got - want)[fine], (2.0 ** -8 * (np.abs(want) + mag) + 2.0 ** -10 * mag)[fine]
    worst = float((err / np.maximum(bar, 1e-30)).max()) if err.size else 0.0
    say(f"  {tag}: worst error / bound {worst:.3f}")
    assert worst <= 1.0, tag


def check_decode(s, tag, ref=None, workspace=None, max_ctx=None, **kw):
    import torch
    from paper_2608_22788_amd import binding
    say(tag, kw)
    want, mag = ref or decode_reference(s)
    n = s["q4"].numel()
    full = torch.full((n + 128,), CANARY, dtype=torch.int16, device="cuda")
    out = full[64:64 + n].view(torch.bfloat16).view(s["q4"].shape)
    ws = binding.decode_attn_kv8(s["q4"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["ql"], out,
                                 s["scale"], workspace=workspace, max_ctx_len=max_ctx or s["max_ctx"], **kw)
    torch.cuda.synchronize()
    raw, got = full.cpu().numpy(), f64(out)
    assert (raw[:64] == CANARY).all() and (raw[-64:] == CANARY).all(), "guard band written"
    raw = raw[64:-64].reshape(got.shape)
    for b, q in enumerate(s["ql"].tolist()):
        assert (raw[b, q:] == CANARY).all(), f"padded rows of sequence {b} written"
    within(np.concatenate([got[b, :q] for b, q in enumerate(s["ql"].tolist())]), want, mag, tag)
    assert int(ws[:1 << 20].count_nonzero()) == 0, "counters left set"
    return out


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_partition_edges(case):
    from paper_2608_22788_amd import binding
    name, Hq, Hkv, D, qmax, ql, cl, _ = case
    s = make8((Hq, Hkv, D), ql, [max(n, q) for n, q in zip(cl, ql)], seed=7, qmax=qmax)
    ref = decode_reference(s)
    shape = binding.shape_of(s["q4"], s["k_pages"], s["table"], s["max_ctx"])
    ws = binding.new_workspace(binding.decode_kv8_workspace_size(shape))
    for call in range(2):   # the second call finds the first one's partials and cleared counters
        check_decode(s, f"kv8 {name} call {call}", ref, workspace=ws)
    check_decode(s, f"kv8 {name}", ref, variant=binding.VARIANT_WAVE)
    for workers in (1, 2, 5, 333):
        check_decode(s, f"kv8 {name}", ref, num_workers=workers)


@pytest.mark.parametrize("case", SPARSE, ids=[c[0] for c in SPARSE])
def test_fewer_pages_than_workers(case):
    name, Hq, Hkv, D, qmax, ql, cl, bound, _ = case
    import torch
    s = make8((Hq, Hkv, D), ql, [max(n, q) for n, q in zip(cl, ql)], seed=9, qmax=qmax)
    B, have = s["table"].shape
    need = (bound + 15) // 16
    s["table"] = torch.cat((s["table"], torch.full((B, max(0, need - have)), -5, dtype=torch.int32, device="cuda")), 1).contiguous()
    check_decode(s, f"kv8 sparse {name}", max_ctx=bound)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 128), (64, 4, 128), (8, 2, 64), (6, 2, 64), (10, 2, 128), (7, 1, 64)],
                         ids=str)
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 65, 200])
def test_lengths(heads, length):
    """Every row count that a unit can have, behind contexts that end in every part of a step."""
    G = heads[0] // heads[1]
    for qmax in {1, 2, min(16, 32 // G), min(16, 64 // G)}:
        ql = [min(qmax, length), 1, min(max(qmax // 2, 1), length)]
        s = make8(heads, ql, [length, length, length + 16], seed=length, qmax=qmax)
        check_decode(s, f"kv8 {heads} length {length} q {ql}")


@pytest.mark.parametrize("heads", [(32, 8, 128), (64, 4, 128), (8, 2, 64), (16, 1, 64)], ids=str)
@pytest.mark.parametrize("qmax", [1, 3, 4])
def test_values_that_a_row_does_not_see(heads, qmax):
    """NaN codes of keys and values of the draft block: rows in front of them do
    not see them."""
    import torch
    ql = [qmax, qmax, 1, qmax]
    s = make8(heads, ql, [100, 33 + qmax, 50, 700], seed=3, qmax=qmax)
    table = s["table"].cpu().numpy()

    def plant(name, b, t, g, d):
        s[name].view(torch.uint8)[int(table[b, t // 16]), g, t % 16, d] = NAN

    g = heads[1] - 1
    plant("v_pages", 0, 99, 0, 5)
    plant("v_pages", 0, 97, g, 40)
    plant("v_pages", 0, 98, g, slice(8, 11))
    plant("k_pages", 0, 99, g, 6)
    plant("v_pages", 1, 33, 0, slice(0, heads[2]))
    plant("v_pages", 3, 100, g, 1)              # seen by every row
    plant("k_pages", 3, 699, 0, slice(0, 2))
    ref = decode_reference(s)
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
    for workers in (0, 3, 50):
        check_decode(s, f"kv8 NaN {heads}", ref, num_workers=workers)


def test_powers_of_any_size():
    """Powers that differ by far between pages, and by a whole page's worth of keys."""
    s = make8((32, 8, 128), [4, 1], [900, 70], seed=4)
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    b = s["scales"].view(torch.uint8)
    b[..., 0] = torch.randint(100, 120, b.shape[:2], generator=g, device="cuda").to(torch.uint8)
    b[..., 1] = torch.randint(27, 228, b.shape[:2], generator=g, device="cuda").to(torch.uint8)
    check_decode(s, "kv8 powers")


def test_many_sequences():
    rng = np.random.default_rng(2)
    n = 700
    ql = rng.integers(0, 3, n).tolist()
    s = make8((8, 2, 64), ql, [max(q, int(x)) for q, x in zip(ql, rng.integers(0, 90, n))], seed=5)
    check_decode(s, "kv8 700 sequences")
    s = make8((4, 1, 128), [1] * 4096, rng.integers(1, 40, 4096).tolist(), seed=6)
    check_decode(s, "kv8 4096 sequences")


def test_pages_behind_4_gib():
    """Offsets of pages and powers that pass 32 bits."""
    import torch
    s = make8((32, 8, 128), [2, 1], [150, 40], seed=8)
    table, n = s["table"].long(), s["k_pages"].shape[0]
    pages = 300000                       # 4.9 GB of codes each
    place = torch.randperm(pages - 262200, device="cuda")[:n] + 262200     # behind 4 GiB
    for name in ("k_pages", "v_pages"):
        far = torch.empty(pages, *s[name].shape[1:], dtype=torch.float8_e4m3fn, device="cuda")
        far.view(torch.uint8)[place] = s[name].view(torch.uint8)
        s[name + "_near"], s[name] = s[name], far
    scales = torch.empty(pages, *s["scales"].shape[1:], dtype=torch.float8_e8m0fnu, device="cuda")
    scales.view(torch.uint8)[place] = s["scales"].view(torch.uint8)
    near = dict(s, k_pages=s["k_pages_near"], v_pages=s["v_pages_near"])
    ref = decode_reference(near)
    s["scales"], s["table"] = scales, torch.where(table >= 0, place[table.clamp(min=0)], table).to(torch.int32).contiguous()
    check_decode(s, "kv8 far pages", ref)


def largest_power(s, seen_by_all, byte=246):
    """The last page of every sequence at the largest power that a cache may have:
    codes of zero for the tokens that all rows see (`seen_by_all` of each sequence),
    +-448 for the others and for the slots behind the last token."""
    import torch
    for b, n in enumerate(s["ctx"].tolist()):
        pid = int(s["table"][b, (n - 1) // 16])
        s["scales"].view(torch.uint8)[pid] = byte
        for k, name in enumerate(("k_pages", "v_pages")):
            codes = s[name].view(torch.uint8)[pid]
            codes[:] = 0
            first = max(seen_by_all[b] - (n - 1) // 16 * 16, 0)
            codes[:, first:, ::2], codes[:, first:, 1::2] = (0x7e, 0xfe) if k else (0xfe, 0x7e)


@pytest.mark.parametrize("heads", [(32, 8, 128), (64, 4, 128), (8, 2, 64), (16, 1, 64)], ids=str)
@pytest.mark.parametrize("qmax", [1, 4])
def test_the_largest_power(heads, qmax):
    """Rows that do not see values of 448 times the largest power, the largest finite
    ones of bf16, are as without them."""
    s = make8(heads, [qmax, qmax, 1], [100, 20 + qmax, 900], seed=11, qmax=qmax)
    largest_power(s, [n - q + 1 for n, q in zip(s["ctx"].tolist(), s["ql"].tolist())])
    from paper_2608_22788_amd import binding
    import torch
    want, mag = decode_reference(s)
    first = np.concatenate(([0], np.cumsum(s["ql"].cpu().numpy())))[:-1]   # the rows that see none
    for workers in (0, 1, 3, 50):
        out = torch.zeros_like(s["q4"])
        binding.decode_attn_kv8(s["q4"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["ql"], out,
                                s["scale"], max_ctx_len=s["max_ctx"], num_workers=workers)
        within(f64(out)[:, 0], want[first], mag[first], f"kv8 largest power {heads} workers {workers}")
