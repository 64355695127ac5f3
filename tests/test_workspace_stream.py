"""Calls that are given a stream and no workspace make theirs on that stream:
memory that the allocator ties to another one may still be in use there, or be
handed out there again while the call runs.  Shown without a GPU, with the
library's calls and torch's allocations recorded."""
import contextlib

import pytest
import torch

from paper_2608_22788_amd import binding


class Side:
    cuda_stream = 0x1234


class Foreign:
    cuda_stream = 0x5678


@pytest.fixture
def recorded(monkeypatch):
    """The streams under which workspaces were made, and whether they were
    zeroed there."""
    current, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream if stream is not None else current[0]
        try:
            yield
        finally:
            current[0] = before

    def recording(kind):
        make = getattr(torch, kind)

        def f(*a, **kw):
            if kw.get("dtype") is torch.uint8:
                made.append((kind, current[0]))
            return make(*a, **kw)
        return f

    class Lib:
        launched = []

        def __getattr__(self, name):
            if name.endswith("_workspace_size"):
                return lambda *a: 512
            return lambda *a: self.launched.append((name, a)) or 0

    lib = Lib()
    lib.launched = []
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Stream", Side)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device: ("external", ptr))
    for kind in ("empty", "zeros"):
        monkeypatch.setattr(torch, kind, recording(kind))
    monkeypatch.setattr(binding, "lib", lib)
    monkeypatch.setattr(binding, "_check_device", lambda *t, **kw: None)
    monkeypatch.setattr(binding, "_check_tensors", lambda *t: None)
    monkeypatch.setattr(binding, "_stream_ptr", lambda s: 0 if s is None else s.cuda_stream)
    return made, lib.launched


def bf(*shape):
    return torch.ones(*shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.ones(*shape, dtype=torch.int32)


def decode(stream, **kw):
    return binding.decode_attn(bf(2, 1, 4, 64), bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(2, 2), i32(2), i32(2),
                               bf(2, 1, 4, 64), 1.0, stream=stream, **kw)


def accept(stream, **kw):
    return binding.spec_accept(torch.ones(2, 3, 5), None, i32(2, 2), i32(2), torch.ones(2, 2), torch.ones(2), i32(2), i32(2),
                               stream=stream, **kw)


def chunk(stream, **kw):
    return binding.chunk_attn(bf(5, 4, 64), bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(2, 2), i32(2), i32(3), bf(5, 4, 64), 1.0,
                              stream=stream, **kw)


def draw(stream, **kw):
    return binding.sample(torch.ones(2, 8), torch.ones(2), i32(2), stream=stream, **kw)


@pytest.mark.parametrize("call, kind", [(decode, "zeros"), (accept, "empty"), (chunk, "empty"), (draw, "empty")],
                         ids=["decode_attn", "spec_accept", "chunk_attn", "sample"])
def test_workspace_is_made_on_the_calls_stream(recorded, call, kind):
    made, launched = recorded
    side = Side()
    ws = call(side)
    assert made == [(kind, side)]
    assert launched[-1][1][-1] == side.cuda_stream and ws.data_ptr() in launched[-1][1]
    call(None)                                # the current stream, as before
    assert made[1:] == [(kind, None)]
    del made[:]
    call(Foreign())                           # a stream object of another library
    assert made == [(kind, ("external", Foreign.cuda_stream))]
    own = torch.ones(4096, dtype=torch.uint8)
    del made[:]
    assert call(side, workspace=own) is own and not made


@pytest.mark.parametrize("call", [decode, accept, chunk, draw], ids=["decode_attn", "spec_accept", "chunk_attn", "sample"])
def test_workspace_that_repeats_its_memory_is_refused(recorded, call):
    """It has as many elements as the call needs bytes, and a single byte."""
    _, launched = recorded
    with pytest.raises(ValueError):
        call(None, workspace=torch.ones(1, dtype=torch.uint8).expand(1 << 20))
    assert not launched
