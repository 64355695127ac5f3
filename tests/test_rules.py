"""Rules on logits without a GPU: refusals before any HIP call, and the oracle
against hand-worked rows."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rules as orc
from paper_2608_22788_amd import binding as b


def config(**kw):
    d = dict(num_seqs=2, vocab=100, logits_type=0, out_type=0, max_tokens=10, num_biases=5, row_stride=100,
             out_stride=100, token_stride=10, allowed_stride=4)
    d.update(kw)
    return b.RulesConfig(*(d[f] for f, _ in b.RulesConfig._fields_))


def rules(cfg, logits=16, out=4096, tokens=16, lens=16, prompt=16, rep=16, freq=16, pres=16, starts=16, ids=16,
          values=16, allowed=16):
    return b.lib.ts_logit_rules(ctypes.byref(cfg) if cfg else None, logits, out, tokens, lens, prompt, rep, freq, pres,
                                starts, ids, values, allowed, None)


@pytest.mark.parametrize("kw", [dict(num_seqs=0), dict(num_seqs=65537), dict(vocab=0), dict(vocab=(1 << 20) + 1)],
                         ids=str)
def test_bad_shapes_rejected(kw):
    assert rules(config(**kw)) == -2 and b.lib.ts_last_error()


@pytest.mark.parametrize("kw", [
    dict(logits_type=2), dict(out_type=-1), dict(row_stride=99), dict(out_stride=99), dict(row_stride=1 << 41),
    dict(max_tokens=-1), dict(max_tokens=(1 << 29) + 1), dict(token_stride=9), dict(num_biases=-1),
    dict(num_biases=(1 << 30) + 1), dict(allowed_stride=3)], ids=str)
def test_bad_arguments_rejected(kw):
    assert rules(config(**kw)) == -6 and b.lib.ts_last_error()


def test_pointers_rejected():
    assert rules(None) == -1
    assert rules(config(), logits=None) == -1 and rules(config(), out=None) == -1
    assert rules(config(), tokens=None) == -1 and rules(config(), lens=None) == -1
    assert rules(config(), tokens=None, rep=None, freq=None, pres=None) == -1      # lengths of nothing
    for name in ("starts", "ids", "values"):
        assert rules(config(), **{name: None}) == -1
    for name in ("logits", "out", "tokens", "lens", "prompt", "rep", "freq", "pres", "starts", "ids", "values", "allowed"):
        assert rules(config(), **{name: 4098}) == -6, name
    assert rules(config(logits_type=1), logits=17) == -6
    assert rules(config(), out=16) != -6 or "equal" not in b.lib.ts_last_error().decode()
    assert rules(config(out_type=1), out=16) == -6 and rules(config(out_stride=104), out=16) == -6


def test_binding_refuses_other_tensors():
    f, i = torch.zeros, lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    good = dict(logits=f(2, 100), out=f(2, 100), tokens=i(2, 7), lens=i(2), prompt_lens=i(2), repetition=f(2),
                frequency=f(2), presence=f(2), bias_starts=i(3), bias_tokens=i(4), bias_values=f(4), allowed=i(2, 4))
    for name, bad in (("logits", f(2, 100).double()), ("logits", f(100, 2).T), ("out", f(2, 99)), ("out", f(2, 100).half()),
                      ("tokens", i(3, 7)), ("tokens", i(7, 2).T), ("tokens", f(2, 7)), ("lens", i(3)), ("prompt_lens", f(2)),
                      ("repetition", i(2)), ("frequency", f(4)[::2]), ("presence", f(1)), ("bias_starts", i(2)),
                      ("bias_tokens", i(5)), ("bias_values", None), ("allowed", i(2, 3)), ("allowed", f(2, 4))):
        with pytest.raises(ValueError, match=name):
            b.logit_rules(**{**good, name: bad})
    with pytest.raises(ValueError, match="CUDA"):
        b.logit_rules(**good)


def test_oracle_by_hand():
    l = np.array([[2.0, -2.0, 0.5, 1.0, -np.inf, 3.0]])
    tokens = np.array([[0, 1, 2, 2, 2, 4, 9, -1, 5]])
    kw = dict(tokens=tokens, lens=[8], prompt_lens=[2], repetition=[2.0], frequency=[0.25], presence=[0.5])
    x, _ = orc.row(l[0], 0, **kw)
    # prompt 0, 1; answer 2 three times and 4; 5 lies behind the length
    assert x.tolist() == [1.0, -4.0, 0.25 - 0.75 - 0.5, 1.0, -np.inf, 3.0]
    x, _ = orc.row(l[0], 0, bias_starts=[1, 5], bias_tokens=[0, 3, 3, 1, 77], bias_values=[9, 1.0, -3.0, -np.inf, 1.0])
    assert x.tolist() == [2.0, -np.inf, 0.5, -1.0, -np.inf, 3.0]
    x, _ = orc.row(l[0], 0, allowed=np.array([[0b101001]]))
    assert x.tolist() == [2.0, -np.inf, -np.inf, 1.0, -np.inf, 3.0]
    kw.update(repetition=[-1.0], frequency=[np.nan], presence=[np.inf])
    assert orc.row(l[0], 0, **kw)[0].tolist() == l[0].tolist()
