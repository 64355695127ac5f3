"""Sampling without a GPU: refusals before any HIP call, and the float64 oracle
against hand-worked cases."""
import ctypes

import numpy as np
import pytest

from oracle import chunk as orc
from paper_2608_22788_amd import binding as b


def call(B=4, V=100, kind=0, logits=16, stride=100, temperature=None, k=None, p=None, m=None, u=16, token=16,
         logprob=None, ws=256, nbytes=1 << 40):
    return b.lib.ts_sample(B, V, kind, logits, stride, temperature, k, p, m, u, token, logprob, ws, nbytes, None)


def test_refusals():
    need = b.sample_workspace_size(4, 100)
    assert need > 0 and need % 256 == 0
    for kw in (dict(B=0), dict(B=65537), dict(V=0), dict(V=(1 << 20) + 1, stride=1 << 21), dict(kind=2), dict(kind=-1),
               dict(stride=99), dict(stride=(1 << 32) + 1), dict(logits=18), dict(logits=17, kind=1), dict(ws=128)):
        assert call(**kw) == -6, kw
        assert b.lib.ts_last_error()
    for name in ("logits", "u", "token", "ws"):
        assert call(**{name: None}) == -1, name
    assert call(nbytes=need - 1) == -3
    for B, V in ((0, 5), (5, 0), (70000, 5), (5, 1 << 21)):
        assert b.lib.ts_sample_workspace_size(B, V) == 0
        with pytest.raises(b.TsError):
            b.sample_workspace_size(B, V)


def test_binding_checks_its_tensors():
    import torch
    x, u, t = torch.zeros(2, 8), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for bad in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.t()), dict(u=u.double()), dict(u=u[:1]),
                dict(token=t.long()), dict(top_k=u), dict(top_p=t), dict(temperature=torch.zeros(3)),
                dict(min_p=torch.zeros(4)[::2]), dict()):            # the last: not on a GPU
        kw = dict(logits=x, u=u, token=t)
        kw.update(bad)
        with pytest.raises(ValueError):
            b.sample(kw.pop("logits"), kw.pop("u"), kw.pop("token"), **kw)


def test_oracle_filters():
    row = np.log(np.array([0.1, 0.4, 0.1, 0.3, 0.1]))
    ids = lambda **f: list(orc.kept_tokens(row, **f)[0])  # noqa: E731
    assert ids() == [0, 1, 2, 3, 4]
    assert ids(top_k=3) == [0, 1, 3]              # of equal ones the lowest index
    assert ids(top_p=0.6) == [1, 3]
    assert ids(top_p=0.39) == [1] and ids(top_p=0.0) == [1]
    assert ids(min_p=0.5) == [1, 3] and ids(min_p=1.0) == [1]
    assert ids(top_k=2, top_p=0.6) == [1, 3]      # 0.4 / 0.7 is below 0.6
    assert ids(top_k=2, top_p=0.5) == [1]
    assert ids(temperature=0.0) == [1]
    flat = np.zeros(4)
    assert list(orc.kept_tokens(flat, top_p=0.5)[0]) == [0, 1]     # nothing kept beyond half of the mass


def test_oracle_draw():
    row = np.array([0.0, -np.inf, 0.0, np.nan])
    assert orc.sample(row, 0.0) == (0, np.log(0.5))
    assert orc.sample(row, 0.49)[0] == 0 and orc.sample(row, 0.5)[0] == 2 and orc.sample(row, 5.0)[0] == 2
    assert orc.sample(np.full(3, -np.inf), 0.5) == (-1, -np.inf)
    assert orc.sample(row, 0.9, temperature=0.0) == (0, 0.0)
    assert ctypes.sizeof(b.ChunkShape) == 48 and ctypes.sizeof(b.RopeConfig) == 48
