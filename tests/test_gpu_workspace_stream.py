"""Calls on another stream that make their own workspace: memory that work
queued on the current stream still writes, or that the current stream is handed
as soon as the returned workspace is dropped, is not theirs."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_chunk import make

pytestmark = pytest.mark.gpu


def calls():
    """name -> (workspace bytes, call(**kw), outputs), on inputs that are ready."""
    import torch
    from paper_2608_22788_amd import binding as b
    out = {}
    s = make(32, 8, 128, [300, 1, 20], [2000, 3000, 0], seed=1)
    o = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    out["chunk_attn"] = (b.chunk_workspace_size(b.chunk_shape_of(s["q"], s["k_pages"], s["table"])),
                         lambda **kw: b.chunk_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["ctx"], s["starts"], o,
                                                   s["scale"], **kw), (o,))
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn(16, 50257, generator=g, device="cuda")
    u, top_p = torch.rand(16, generator=g, device="cuda"), torch.full((16,), 0.9, device="cuda")
    token, lp = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.zeros(16, device="cuda")
    out["sample"] = (b.sample_workspace_size(16, 50257),
                     lambda **kw: b.sample(logits, u, token, lp, top_p=top_p, **kw), (token, lp))
    d = make(32, 8, 128, [1] * 4, [3000, 20, 700, 5000], seed=3)
    q, table, lens = d["q"].contiguous().view(4, 1, 32, 128), d["table"].clamp(min=0), torch.ones(4, dtype=torch.int32, device="cuda")
    do = torch.zeros_like(q)
    out["decode_attn"] = (b.workspace_size(b.shape_of(q, d["k_pages"], table)),
                          lambda **kw: b.decode_attn(q, d["k_pages"], d["v_pages"], table, d["ctx"], lens, do, d["scale"], **kw),
                          (do,))
    p = torch.softmax(torch.randn(8, 5, 50257, generator=g, device="cuda"), -1)
    pd = torch.softmax(torch.randn(8, 4, 50257, generator=g, device="cuda"), -1)
    draft = torch.randint(0, 50257, (8, 4), generator=g, device="cuda", dtype=torch.int32)
    n = torch.full((8,), 4, dtype=torch.int32, device="cuda")
    ua, us = torch.rand(8, 4, generator=g, device="cuda"), torch.rand(8, generator=g, device="cuda")
    acc, nxt = (torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(2))
    out["spec_accept"] = (int(b.lib.ts_spec_accept_workspace_size(8, 50257)),
                          lambda **kw: b.spec_accept(p, pd, draft, n, ua, us, acc, nxt, **kw), (acc, nxt))
    return out


@pytest.mark.parametrize("name", ["chunk_attn", "sample", "decode_attn", "spec_accept"])
def test_workspace_of_a_call_on_another_stream(name):
    import torch
    nbytes, call, outputs = calls()[name]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    side = torch.cuda.Stream()
    wrapped = type("Handle", (), {"cuda_stream": side.cuda_stream})()     # another library's stream object
    for rep, stream in enumerate((side, side, side, wrapped)):
        say(name, "repetition", rep)
        for t in outputs:
            t.zero_()
        before = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for i in range(200):                    # still running when the call begins
            before.fill_(i)
        del before
        ws = call(stream=stream)
        del ws
        after = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        for i in range(200):                    # while the call runs, and behind it
            after.fill_(i)
        torch.cuda.synchronize()
        for got, ref in zip(outputs, want):
            assert np.array_equal(got.cpu().view(torch.uint8).numpy(), ref.cpu().view(torch.uint8).numpy())
