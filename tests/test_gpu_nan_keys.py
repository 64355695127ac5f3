"""A NaN among the keys that a row sees makes the whole row NaN, wherever its keys
are split and however the pieces meet; rows that do not see it are as without it.
Every kernel of ts_decode_attn, against oracle/chunk.py, with the tolerances of
test_gpu_chunk.py (weights are rounded to bf16 here too)."""
import numpy as np
import pytest

from gpu_util import say
from oracle import chunk as orc
from test_gpu_chunk import f64, make
from test_gpu_group import CASES
from test_gpu_kv8_decode import within

pytestmark = pytest.mark.gpu

VALU, TEAM = 3, 2


def inputs(heads, q_lens, ctx, qmax, seed):
    import torch
    s = make(*heads, q_lens, [n - q for n, q in zip(ctx, q_lens)], seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    s["q4"] = torch.empty(len(q_lens), qmax, heads[0], heads[2], dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    s["ql"] = torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    return s


def reference(s):
    q, ql = f64(s["q4"]), s["ql"].cpu().numpy()
    return orc.chunk_attention(np.concatenate([q[b, :n] for b, n in enumerate(ql)]), f64(s["k_pages"]), f64(s["v_pages"]),
                               s["table"].cpu().numpy(), s["ctx"].cpu().numpy(), np.concatenate(([0], np.cumsum(ql))),
                               s["scale"])


def check(s, ref, tag, variant=0, workers=0):
    import torch
    from paper_2608_22788_amd import binding
    say(tag, "variant", variant, "workers", workers)
    out = torch.zeros_like(s["q4"])
    ws = binding.decode_attn(s["q4"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["ql"], out, s["scale"],
                             max_ctx_len=s["max_ctx"], variant=variant, num_workers=workers)
    torch.cuda.synchronize()
    got = f64(out)
    within(np.concatenate([got[b, :n] for b, n in enumerate(s["ql"].tolist())]), *ref, tag)
    assert int(ws[:1 << 20].count_nonzero()) == 0, "counters left set"


ROWS64 = ("rows64", 32, 8, 128, 16, [16, 3, 16], [4000, 300, 17], None)


@pytest.mark.parametrize("case", [*CASES, ROWS64], ids=[*(c[0] for c in CASES), "rows64"])
def test_nan_keys(case):
    """A key near each sequence's start, one in its middle, and the last row's own."""
    name, Hq, Hkv, D, qmax, ql, cl, _ = case
    cl = [max(n, q) for n, q in zip(cl, ql)]
    s = inputs((Hq, Hkv, D), ql, cl, qmax, seed=17)
    table = s["table"].cpu().numpy()
    for b, n in enumerate(cl):
        t = (min(3, n - 1), n // 2, n - 1)[b % 3]
        s["k_pages"][int(table[b, t // 16]), b % Hkv, t % 16, (11 * b) % D] = float("nan")
    ref = reference(s)
    assert np.isnan(ref[0]).any()
    variants = [0, 1] + ([TEAM] if D == 128 else []) + ([VALU] if qmax == 1 and Hq // Hkv in (1, 2, 4, 8) else [])
    for variant in variants:
        for workers in (0, 1, 5, 64):
            check(s, ref, f"NaN keys {name}", variant, workers)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] in ("short_long", "merge_kernel", "last", "d64_3")] + [ROWS64],
                         ids=lambda c: c[0])
def test_nan_queries(case):
    name, Hq, Hkv, D, qmax, ql, cl, _ = case
    s = inputs((Hq, Hkv, D), ql, [max(n, q) for n, q in zip(cl, ql)], qmax, seed=18)
    for b, q in enumerate(ql):
        if q > 0:
            s["q4"][b, q - 1, (3 * b) % Hq, (7 * b) % D] = float("nan")
    ref = reference(s)
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
    for variant in [0, 1] + ([TEAM] if D == 128 else []) + ([VALU] if qmax == 1 else []):
        for workers in (0, 5):
            check(s, ref, f"NaN queries {name}", variant, workers)
