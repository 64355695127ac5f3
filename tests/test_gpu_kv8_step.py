"""A serving step over the cache held in 8 bits as a replica runs it: a prompt's
append and attention, then decoding token by token, penalties and masks on the
logits and the draw; against the float64 oracles, captured into graphs that share
a workspace, on two streams, and next to each other."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import chunk as orc
from oracle import rules
from test_gpu_chunk import f64
from test_gpu_kv8_append import inputs
from test_gpu_kv8_decode import reference8, within

pytestmark = pytest.mark.gpu

VOCAB = 5000


def step_inputs(seed, q_lens, past, heads=(8, 2, 128)):
    from paper_2608_22788_amd import binding
    s = inputs(heads, (q_lens, past), heads[2], "both", seed=seed)
    for name in ("k_pages", "v_pages"):      # whole pages of numbers
        u = s[name].view(torch.uint8)
        u[(u & 127) == 127] = 0x38
    g = torch.Generator(device="cuda").manual_seed(seed)
    B = len(q_lens)
    s["q_rot"], s["out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["q"])
    s["head"] = torch.randn(heads[0] * heads[2], VOCAB, generator=g, device="cuda") * 0.2
    s["last"] = (s["starts"][1:] - 1).long()
    s["u"] = torch.rand(B, generator=g, device="cuda")
    s["text"] = torch.randint(0, 200, (B, 60), generator=g, device="cuda", dtype=torch.int32)
    s["lens"] = torch.randint(0, 61, (B,), generator=g, device="cuda", dtype=torch.int32)
    s["rep"] = 1.0 + torch.rand(B, generator=g, device="cuda")
    s["freq"] = torch.rand(B, generator=g, device="cuda")
    s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (B, (VOCAB + 31) // 32), generator=g, device="cuda").to(torch.int32)
    s["allowed"][0] = 0                      # a grammar that allows nothing
    s["token"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.zeros(B, device="cuda")
    s["logits"] = torch.zeros(B, VOCAB, device="cuda")
    s["ruled"] = torch.zeros(B, VOCAB, device="cuda")
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])
    s["ws"] = torch.empty(binding.chunk_kv8_workspace_size(shape), dtype=torch.uint8, device="cuda")
    s["sample_ws"] = torch.empty(binding.sample_workspace_size(B, VOCAB), dtype=torch.uint8, device="cuda")
    return s


def attend(s, stream=None):
    from paper_2608_22788_amd import binding
    binding.rope_append_kv8(s["q"], s["k"], s["v"], s["q_rot"], s["k_pages"], s["v_pages"], s["scales"], s["table"],
                            s["ctx"], s["starts"], s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"], stream=stream)
    binding.chunk_attn_kv8(s["q_rot"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["starts"],
                           s["out"], s["scale"], workspace=s["ws"], max_q_len=s["max_q"], max_ctx_len=s["max_ctx"],
                           stream=stream)


def draw(s, stream=None):
    from paper_2608_22788_amd import binding
    binding.logit_rules(s["logits"], s["ruled"], tokens=s["text"], lens=s["lens"], repetition=s["rep"],
                        frequency=s["freq"], allowed=s["allowed"], stream=stream)
    binding.sample(s["ruled"], s["u"], s["token"], s["logprob"], workspace=s["sample_ws"], stream=stream)


def product(s):
    s["logits"].copy_(torch.mm(s["out"][s["last"]].float().flatten(1), s["head"]))


MIXED = ([70, 1, 1, 33, 2, 5], [200, 900, 15, 0, 60, 1])


def test_step_against_the_oracles():
    s = step_inputs(1, *MIXED)
    say("step")
    attend(s)
    product(s)
    draw(s)
    torch.cuda.synchronize()
    want, mag = reference8(s, f64(s["q_rot"]), s["starts"].cpu().numpy())
    used = ~np.isnan(want).all(axis=(1, 2))
    within(f64(s["out"])[used], want[used], mag[used], "attention of the step")
    logits, ruled = s["logits"].cpu().numpy(), s["ruled"].cpu().numpy()
    for b in range(len(MIXED[0])):
        x, size = rules.row(logits[b], b, tokens=s["text"].cpu().numpy(), lens=s["lens"].tolist(),
                            repetition=s["rep"].tolist(), frequency=s["freq"].tolist(), allowed=s["allowed"].cpu().numpy())
        open_ = np.isfinite(x)
        assert np.array_equal(open_, np.isfinite(ruled[b]))
        assert (np.abs(ruled[b] - np.where(open_, x, 0))[open_] <= 2.0 ** -18 * size[open_]).all()
        token, lp = orc.sample(ruled[b], s["u"][b].item())
        assert int(s["token"][b]) == token
        assert token == -1 or (open_[token] and abs(float(s["logprob"][b]) - lp) < 1e-5)
    assert int(s["token"][0]) == -1


def test_a_prompt_then_tokens_one_by_one():
    """The cache that a prompt and thirty decoding steps leave, read by decode and by
    chunk attention, against the oracle on its codes."""
    from paper_2608_22788_amd import binding
    heads, steps = (8, 2, 64), 30
    s = step_inputs(7, [50, 3, 20], [0, 40, 5], heads=heads)
    B = 3
    room = int(s["ctx"].max()) // 16 + 4
    s["table"] = torch.randperm(B * room, device="cuda")[:B * room].view(B, room).to(torch.int32).contiguous()
    n = B * room
    s["k_pages"] = torch.full((n, 2, 16, 64), 0x38, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    s["v_pages"] = s["k_pages"].clone()
    s["scales"] = torch.full((n, 2, 2), 120, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    s["max_ctx"] = room * 16
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])
    s["ws"] = torch.empty(binding.chunk_kv8_workspace_size(shape), dtype=torch.uint8, device="cuda")
    attend(s)
    one = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    ones = torch.ones(B, dtype=torch.int32, device="cuda")
    q, k, v = (torch.empty(B, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    turned, a, b = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    ws = None
    for step in range(steps):
        say("token", step)
        for t in (q, k, v):
            t.normal_().mul_(1.0 + step / 10)
        s["ctx"] += 1
        binding.rope_append_kv8(q, k, v, turned, s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], one,
                                s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"])
        ws = binding.decode_attn_kv8(turned.view(B, 1, 8, 64), s["k_pages"], s["v_pages"], s["scales"], s["table"],
                                     s["ctx"], ones, a.view(B, 1, 8, 64), s["scale"], workspace=ws, max_ctx_len=s["max_ctx"])
        binding.chunk_attn_kv8(turned, s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], one, b, s["scale"])
        torch.cuda.synchronize()
        want, mag = reference8(s, f64(turned), one.cpu().numpy())
        within(f64(a), want, mag, "decode")
        within(f64(b), want, mag, "chunk")


def test_step_captured_and_replayed():
    """Graphs of two steps that share their workspaces, replayed in turn with eager
    work between, give the eager results bit for bit every time."""
    steps = [step_inputs(2, *MIXED), step_inputs(3, [1] * 6, [40, 700, 5, 90, 1000, 15])]
    big = max((s["ws"] for s in steps), key=lambda t: t.numel())
    for s in steps:
        s["ws"], s["sample_ws"] = big, steps[0]["sample_ws"]
    names = ("q_rot", "k_pages", "v_pages", "scales", "out", "ruled", "token", "logprob")
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    refs, graphs, caches = [], [], []
    for s in steps:
        caches.append({k: s[k].clone() for k in ("k_pages", "v_pages", "scales")})
        attend(s)
        product(s)
        draw(s)
        torch.cuda.synchronize()
        refs.append({k: s[k].clone() for k in names})
    side = torch.cuda.Stream()
    for s in steps:
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                attend(s)
                draw(s)
        graphs.append(g)
        torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        say("replay", rep)
        for s, c in zip(steps, caches):     # eager work between replays
            for k, t in c.items():
                bits(s[k]).copy_(bits(t))
            for k in ("q_rot", "out", "ruled", "token", "logprob"):
                s[k].fill_(3)
        big.fill_(rep * 80)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, ref in zip(steps, refs):
            n = int(s["starts"][-1])
            for name in names:
                rows = slice(0, n if name in ("q_rot", "out") else None)
                assert torch.equal(bits(s[name][rows]), bits(ref[name][rows])), (rep, name)
            assert (s["q_rot"][n:] == 3).all() and (s["out"][n:] == 3).all(), "rows of no sequence were written"


def test_decode_captured_and_replayed_with_a_shared_workspace():
    from paper_2608_22788_amd import binding
    from test_gpu_kv8_decode import make8
    calls = [make8((32, 8, 128), [4, 1, 2], [900, 33, 5000], seed=1), make8((8, 2, 64), [1] * 80, [50 + 7 * i for i in range(80)], seed=2)]
    size = lambda s: binding.decode_kv8_workspace_size(binding.shape_of(s["q4"], s["k_pages"], s["table"], s["max_ctx"]))  # noqa: E731
    ws = binding.new_workspace(max(size(s) for s in calls))
    run = lambda s: binding.decode_attn_kv8(s["q4"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["ql"],  # noqa: E731
                                            s["o"], s["scale"], workspace=ws, max_ctx_len=s["max_ctx"])
    refs, graphs = [], []
    for s in calls:
        s["o"] = torch.zeros_like(s["q4"])
        run(s)
        torch.cuda.synchronize()
        refs.append(s["o"].clone())
    for s in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(s)
        graphs.append(g)
    for rep in range(4):
        say("replay", rep)
        for s in calls:
            s["o"].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, ref in zip(calls, refs):
            assert torch.equal(s["o"], ref), rep


def test_two_streams_with_their_own_workspaces():
    a, b = step_inputs(4, [300, 1, 20], [500, 2000, 0]), step_inputs(5, [1] * 9, [900, 30, 4000] * 3, heads=(32, 4, 128))
    refs = []
    for s in (a, b):
        attend(s)
        product(s)
        draw(s)
        torch.cuda.synchronize()
        refs.append((s["out"].clone(), s["ruled"].clone(), s["token"].clone()))
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for rep in range(5):
        say("two streams, repetition", rep)
        for s in (a, b):
            for k in ("out", "ruled", "token"):
                s[k].zero_()
        torch.cuda.synchronize()
        for s, st in ((a, sa), (b, sb)):
            attend(s, stream=st)
            draw(s, stream=st)
        torch.cuda.synchronize()
        for s, ref in zip((a, b), refs):
            for k, want in zip(("out", "ruled", "token"), ref):
                assert torch.equal(s[k], want), (rep, k)


def test_calls_without_a_workspace_on_a_side_stream():
    from paper_2608_22788_amd import binding
    s = step_inputs(6, [40, 1], [100, 700])
    attend(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros_like(s["out"])
    binding.chunk_attn_kv8(s["q_rot"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["starts"], out,
                           s["scale"], max_q_len=s["max_q"], max_ctx_len=s["max_ctx"], stream=side)
    torch.cuda.synchronize()
    n = int(s["starts"][-1])
    assert torch.equal(out[:n], s["out"][:n])
