"""A serving step around a chunk as a replica runs it -- rotation and append,
attention over the cache, the draw of the next token -- against the float64
oracles, captured into a graph, on two streams, with a cache past 4 GiB, and
next to the library's decode attention."""
import ctypes

import numpy as np
import pytest

from oracle import chunk as orc
from gpu_util import say
from test_gpu_chunk import f64, make

pytestmark = pytest.mark.gpu


def step_inputs(seed, q_lens, past, heads=(8, 2, 128), vocab=5000):
    import torch
    s = make(*heads, q_lens, past, seed=seed, poison=False)
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, _, D = heads
    B = len(q_lens)
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float()
    s["norm"] = (1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    s["q_rot"] = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    s["out"] = torch.zeros_like(s["q_rot"])
    s["head"] = torch.randn(Hq * D, vocab, generator=g, device="cuda") * 0.2
    s["last"] = (s["starts"][1:] - 1).long()
    s["u"] = torch.rand(B, generator=g, device="cuda")
    s["top_p"] = torch.full((B,), 0.9, device="cuda")
    s["token"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.zeros(B, device="cuda")
    from paper_2608_22788_amd import binding
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])
    s["ws"] = torch.empty(binding.chunk_workspace_size(shape), dtype=torch.uint8, device="cuda")
    s["sample_ws"] = torch.empty(binding.sample_workspace_size(B, vocab), dtype=torch.uint8, device="cuda")
    return s


def run_step(s, stream=None):
    from paper_2608_22788_amd import binding
    binding.rope_append(s["q"], s["k"], s["v"], s["q_rot"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"],
                        s["inv_freq"], q_norm=s["norm"], k_norm=s["norm"], stream=stream)
    binding.chunk_attn(s["q_rot"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], s["out"], s["scale"],
                       workspace=s["ws"], max_q_len=s["max_q"], max_ctx_len=s["max_ctx"], stream=stream)


def draw_step(s, stream=None):
    """The model's last product, in plain torch, and the draw."""
    import torch
    from paper_2608_22788_amd import binding
    s["logits"] = torch.mm(s["out"][s["last"]].float().flatten(1), s["head"])
    binding.sample(s["logits"], s["u"], s["token"], s["logprob"], top_p=s["top_p"], workspace=s["sample_ws"], stream=stream)


MIXED = ([70, 1, 1, 33, 0, 5], [200, 900, 15, 0, 60, 1])


def test_step_against_the_oracles():
    import torch
    s = step_inputs(1, *MIXED)
    kp, vp = f64(s["k_pages"]), f64(s["v_pages"])
    num = {k: s[k].cpu().numpy() for k in ("table", "ctx", "starts", "inv_freq")}
    say("step")
    run_step(s)
    draw_step(s)
    torch.cuda.synchronize()
    q, kp, vp = orc.rope_append(f64(s["q"]), f64(s["k"]), f64(s["v"]), kp, vp, num["table"], num["ctx"], num["starts"],
                                num["inv_freq"], f64(s["norm"]), f64(s["norm"]))
    for got, want in ((s["q_rot"], q), (s["k_pages"], kp), (s["v_pages"], vp)):
        assert (np.abs(f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18).all()
    # attention from the rounded q and keys that the kernel had
    want, mag = orc.chunk_attention(f64(s["q_rot"]), f64(s["k_pages"]), f64(s["v_pages"]), num["table"], num["ctx"],
                                    num["starts"], s["scale"])
    # (norms of about 1 leave the inputs' size, so the bound of the attention tests holds)
    assert (np.abs(f64(s["out"]) - want) <= 2.0 ** -8 * (np.abs(want) + mag) + 2.0 ** -10 * mag).all()
    rows = s["logits"].cpu().numpy()
    for b in range(len(MIXED[0])):
        token, lp = orc.sample(rows[b], s["u"][b].item(), top_p=np.float32(0.9))
        assert int(s["token"][b]) == token and abs(float(s["logprob"][b]) - lp) < 1e-5


def test_step_captured_and_replayed():
    """Graphs of two steps that share their workspaces, replayed in turn with
    eager work between, give the eager results bit for bit every time."""
    import torch
    steps = [step_inputs(2, *MIXED), step_inputs(3, [1] * 6, [40, 700, 5, 90, 1000, 15])]
    big = max((s["ws"] for s in steps), key=lambda t: t.numel())
    for s in steps:
        s["ws"], s["sample_ws"] = big, steps[0]["sample_ws"]
    refs, graphs, pages = [], [], []
    names = ("q_rot", "k_pages", "v_pages", "out", "token", "logprob")
    for s in steps:
        pages.append((s["k_pages"].clone(), s["v_pages"].clone()))
        run_step(s)
        draw_step(s)
        torch.cuda.synchronize()
        refs.append({k: s[k].clone() for k in names})
    side = torch.cuda.Stream()
    for s in steps:
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                run_step(s)
                from paper_2608_22788_amd import binding
                binding.sample(s["logits"], s["u"], s["token"], s["logprob"], top_p=s["top_p"], workspace=s["sample_ws"])
        graphs.append(g)
        torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        say("replay", rep)
        for s, (k, v) in zip(steps, pages):     # eager work between replays
            s["k_pages"].copy_(k)
            s["v_pages"].copy_(v)
            for name in ("q_rot", "out", "token", "logprob"):
                s[name].fill_(3)
        big.fill_(rep * 80)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, ref in zip(steps, refs):
            for name in names:
                assert torch.equal(s[name].float(), ref[name].float()), (rep, name)


def test_two_streams_with_their_own_workspaces():
    import torch
    a, b = step_inputs(4, [300, 1, 20], [500, 2000, 0]), step_inputs(5, [1] * 9, [900, 30, 4000] * 3, heads=(32, 4, 128))
    refs = []
    for s in (a, b):
        run_step(s)
        draw_step(s)
        torch.cuda.synchronize()
        refs.append((s["out"].clone(), s["token"].clone()))
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for rep in range(5):
        say("two streams, repetition", rep)
        for s in (a, b):
            s["out"].zero_()
            s["token"].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for s, stream in ((a, sa), (b, sb)):
                run_step(s, stream=stream)
                from paper_2608_22788_amd import binding
                binding.sample(s["logits"], s["u"], s["token"], s["logprob"], top_p=s["top_p"], workspace=s["sample_ws"],
                               stream=stream)
        torch.cuda.synchronize()
        for s, (out, token) in zip((a, b), refs):
            assert torch.equal(s["out"].view(torch.int16), out.view(torch.int16)) and torch.equal(s["token"], token)


def test_workspace_of_another_call():
    """Calls with few tiles, or none at all, that take over the workspace of a
    larger one, and one full of ones."""
    import torch
    from paper_2608_22788_amd import binding
    big = make(8, 2, 128, [500, 60, 1], [3000, 100, 2000], seed=10)
    small = make(8, 2, 128, [3, 0, 1], [0, 0, 90], seed=11)
    W = 100
    shape = binding.chunk_shape_of(big["q"], big["k_pages"], big["table"], num_workers=W)
    ws = torch.full((binding.chunk_workspace_size(shape),), 1, dtype=torch.uint8, device="cuda")

    def run(s, starts):
        out = torch.full(s["q"].shape, 7.0, dtype=torch.bfloat16, device="cuda")
        binding.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], starts, out, s["scale"], workspace=ws,
                           num_workers=W)
        torch.cuda.synchronize()
        return out.view(torch.int16)

    say("no rows, workspace of ones")
    assert (run(small, torch.zeros_like(small["starts"])).view(torch.bfloat16) == 7.0).all()
    first = run(small, small["starts"])
    say("after a larger call")
    run(big, big["starts"])
    assert torch.equal(run(small, small["starts"]), first)
    run(big, big["starts"])
    assert (run(small, torch.zeros_like(small["starts"])).view(torch.bfloat16) == 7.0).all()


def test_chunk_agrees_with_decode_attention():
    """Up to 16 new tokens a sequence both kernels compute the same attention:
    they differ by the rounding of either (each within the bound of its tests)."""
    import torch
    from paper_2608_22788_amd import binding
    q_lens, past = [4, 1, 16, 2], [3000, 17, 100, 0]
    s = make(16, 4, 128, q_lens, past, seed=6)
    out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    binding.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], out, s["scale"])
    B, Qm = 4, 16
    q = torch.zeros(B, Qm, 16, 128, dtype=torch.bfloat16, device="cuda")
    padded = torch.zeros_like(q)
    for b in range(B):
        q[b, :q_lens[b]] = s["q"][int(s["starts"][b]):int(s["starts"][b + 1])]
    lens = torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    table = s["table"].clamp(min=0)
    binding.decode_attn(q, s["k_pages"], s["v_pages"], table, s["ctx"], lens, padded, s["scale"])
    torch.cuda.synchronize()
    for b in range(B):
        x, y = out[int(s["starts"][b]):int(s["starts"][b + 1])].float(), padded[b, :q_lens[b]].float()
        assert (x - y).abs().max().item() <= 0.05 and ((x - y).norm() / y.norm()).item() <= 1e-2


def test_chunk_output_in_place_of_the_queries():
    import torch
    from paper_2608_22788_amd import binding
    for W in (0, 1, 7, 1000):
        s = make(8, 2, 128, [200, 1, 90, 16], [700, 30, 0, 5000], seed=9)
        out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        say("in place, workers", W)
        binding.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], out, s["scale"], num_workers=W)
        n = int(s["starts"][-1])
        binding.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], s["q"], s["scale"], num_workers=W)
        assert torch.equal(s["q"][:n].view(torch.int16), out[:n].view(torch.int16))


def test_cache_past_4_gib():
    """Pages whose byte offset needs more than 32 bits, read and written."""
    import torch
    from paper_2608_22788_amd import binding
    s = step_inputs(7, [70, 1], [300, 2000], heads=(32, 8, 128))
    run_step(s)
    n = s["k_pages"].shape[0]
    total = 150_000                     # x 32 KiB: 4.9 GB
    far = dict(s)
    for name in ("k_pages", "v_pages"):
        far[name] = torch.zeros(total, 8, 16, 128, dtype=torch.bfloat16, device="cuda")
        far[name][total - n:] = step_inputs(7, [70, 1], [300, 2000], heads=(32, 8, 128))[name]
    far["table"] = torch.where(s["table"] >= 0, s["table"] + (total - n), s["table"])
    far["out"] = torch.zeros_like(s["out"])
    run_step(far)
    torch.cuda.synchronize()
    assert torch.equal(far["out"].view(torch.int16), s["out"].view(torch.int16))
    for name in ("k_pages", "v_pages"):
        assert torch.equal(far[name][total - n:].view(torch.int16), s[name].view(torch.int16))


def test_empty_calls_and_refusals_of_the_binding():
    import torch
    from paper_2608_22788_amd import binding
    s = make(8, 2, 64, [3, 2], [5, 6], seed=8)
    none = s["q"][:0]
    binding.chunk_attn(none, s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"] * 0, none, s["scale"])
    binding.rope_append(none, s["k"][:0], s["v"][:0], none, s["k_pages"], s["v_pages"], s["table"], s["ctx"],
                        s["starts"] * 0, None)
    out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    good = dict(q=s["q"], k_pages=s["k_pages"], v_pages=s["v_pages"], page_table=s["table"], ctx_lens=s["ctx"],
                q_starts=s["starts"], out=out)
    for name, bad in (("q", s["q"].float()), ("q", s["q"].transpose(0, 1)), ("out", out[:2]), ("out", out[:, :, :32]),
                      ("v_pages", s["v_pages"][:-1]), ("page_table", s["table"].long()), ("ctx_lens", s["ctx"][:1]),
                      ("q_starts", s["starts"][:-1]), ("ctx_lens", s["ctx"].cpu()), ("k_pages", s["k_pages"].transpose(1, 2))):
        with pytest.raises(ValueError):
            binding.chunk_attn(**{**good, name: bad}, scale=1.0)
    with pytest.raises(ValueError):
        binding.rope_append(s["q"], s["k"], s["v"], out, s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"],
                            torch.zeros(32, dtype=torch.float64, device="cuda"))
    with pytest.raises(binding.TsError) as err:
        binding.chunk_attn(**good, scale=1.0, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert err.value.status == -3
    with pytest.raises(binding.TsError):
        binding.chunk_attn(**good, scale=float("nan"))
    wide = torch.zeros(s["q"].shape[0], 16, 64, dtype=torch.bfloat16, device="cuda")
    shape = binding.chunk_shape_of(s["q"], s["k_pages"], s["table"])
    ws = torch.empty(binding.chunk_workspace_size(shape), dtype=torch.uint8, device="cuda")
    args = [ctypes.byref(shape), wide.data_ptr(), 512, s["k_pages"].data_ptr(), s["v_pages"].data_ptr(), s["table"].data_ptr(),
            s["ctx"].data_ptr(), s["starts"].data_ptr(), wide.data_ptr(), 1024, 1.0, ws.data_ptr(), ws.numel(), None]
    assert binding.lib.ts_chunk_attn(*args) == -6                 # in place with two strides
    with pytest.raises(binding.TsError):
        binding.chunk_attn(**good, scale=1.0, max_q_len=6)        # above the number of rows
    torch.cuda.synchronize()
    assert not out.any()
