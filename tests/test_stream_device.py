"""The calls on packed rows and the draw run on a stream of the device that
their tensors are on, and refuse another device's."""
import pytest
import torch

from paper_2608_22788_amd import binding


class OnDevice:
    """A tensor as the check sees it."""
    is_cuda = True

    def __init__(self, index):
        self.device = f"cuda:{index}"
        self.index = index

    def get_device(self):
        return self.index


def stream_on(index):
    return type("Stream", (), {"device_index": index, "cuda_stream": 16})()


@pytest.fixture
def two_devices(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)


def test_the_check(two_devices):
    here, there = OnDevice(1), OnDevice(0)
    binding._check_device(here, None, here)
    binding._check_device(here, stream=stream_on(1))
    binding._check_device(here, stream=type("Handle", (), {"cuda_stream": 16})())     # says nothing about its device
    for tensors, stream in (((here, there), None), ((there, there), None), ((here,), stream_on(0))):
        with pytest.raises(ValueError):
            binding._check_device(*tensors, stream=stream)


def test_every_call_hands_its_stream_to_the_check(monkeypatch):
    seen = []

    def check(*tensors, stream=None):
        seen.append(stream)
        raise ValueError("stop")

    monkeypatch.setattr(binding, "_check_device", check)
    bf = lambda *s: torch.ones(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.ones(*s, dtype=torch.int32)  # noqa: E731
    paged = (bf(3, 2, 16, 64), bf(3, 2, 16, 64), i32(2, 2), i32(2), i32(3))
    s = stream_on(0)
    for call in (lambda: binding.chunk_attn(bf(5, 4, 64), *paged, bf(5, 4, 64), 1.0, stream=s),
                 lambda: binding.rope_append(bf(5, 4, 64), bf(5, 2, 64), bf(5, 2, 64), bf(5, 4, 64), *paged, None, stream=s),
                 lambda: binding.sample(torch.ones(2, 8), torch.ones(2), i32(2), stream=s)):
        with pytest.raises(ValueError, match="stop"):
            call()
    assert seen == [s] * 3
