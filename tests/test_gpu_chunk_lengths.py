"""Lengths that the page table has no room for, and negative ones: rotation
with append and chunk attention clamp them alike, so that a row is at one
position in both and sees its own key."""
import numpy as np
import pytest

from oracle import chunk as orc
from gpu_util import say
from test_gpu_chunk import check_chunk, check_rope, f64, rope_inputs

pytestmark = pytest.mark.gpu

PAGES = 3                # of every sequence: 48 positions
PAST_THE_TABLE = [48, 49, 64, 2 ** 31 - 1, 60, 48 + 2 ** 20, 47]
NEGATIVE = [48, -1, 0, -(2 ** 31), 3, 48, 1]
Q = [1, 1, 5, 2, 20, 48, 16]


def inputs(heads, ctx, norm="none", seed=0):
    import torch
    s = rope_inputs(heads, (Q, [16 * PAGES - q for q in Q]), heads[2], norm, seed=seed)
    s["table"] = s["table"][:, :PAGES].contiguous()
    s["ctx"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    s["max_ctx"] = 16 * PAGES
    return s


@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128)], ids=str)
@pytest.mark.parametrize("ctx", [PAST_THE_TABLE, NEGATIVE], ids=["past the table", "negative"])
def test_lengths_outside_the_table(heads, ctx):
    for norm, interleaved in (("none", False), ("both", True)):
        check_rope(inputs(heads, ctx, norm, seed=3), interleaved, f"rope lengths {ctx} {norm}")
    for workers in (0, 1, 5):
        check_chunk(inputs(heads, ctx, seed=4), f"chunk lengths {ctx}", workers)


def test_rows_see_their_own_keys():
    """One new token per sequence whose key is its query, far larger than the
    cached ones, behind lengths past the table: its own value comes back."""
    import torch
    from paper_2608_22788_amd import binding
    say("rows see their own keys")
    s = inputs((4, 2, 64), PAST_THE_TABLE, seed=5)
    s["starts"] = torch.arange(len(Q) + 1, dtype=torch.int32, device="cuda")
    n = len(Q)
    for name in ("q", "k", "v"):
        s[name] = s[name][:n].contiguous()
    s["k"].mul_(16.0)
    s["q"] = s["k"].repeat_interleave(2, dim=1).contiguous()
    q, out = torch.zeros_like(s["q"]), torch.zeros_like(s["q"])
    binding.rope_append(s["q"], s["k"], s["v"], q, s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], s["inv_freq"])
    binding.chunk_attn(q, s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], out, s["scale"])
    torch.cuda.synchronize()
    # |k|^2 / 8 is about 16^2 x 64 / 8 = 2,048; another key's score has a spread of 16 x 16 x 8 / 8 / 16 = 16, so no weight
    # but the row's own is left
    assert torch.equal(out, s["v"].repeat_interleave(2, dim=1))
    want = orc.rope_append(f64(s["q"]), f64(s["k"]), f64(s["v"]), f64(s["k_pages"]), f64(s["v_pages"]), s["table"].cpu().numpy(),
                           s["ctx"].cpu().numpy(), s["starts"].cpu().numpy(), s["inv_freq"].cpu().numpy())[0]
    assert (np.abs(f64(q) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -14).all()   # (values 16 times those of check_rope: 2^-18 x 16)
