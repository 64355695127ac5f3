"""The operators over the cache held in 8 bits without a GPU: their refusals
before any HIP call, and the oracle's e4m3 against torch's."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_22788_amd import binding as b
from test_abi import base_shape
from test_chunk import BAD_SHAPES, ROOT, config, shape


def append(s, cfg, q=16, k=16, v=16, out=16, kp=16, vp=16, scales=16, table=16, ctx=16, starts=16, freq=16, qn=None,
           kn=None):
    return b.lib.ts_rope_append_kv8(ctypes.byref(s) if s else None, ctypes.byref(cfg) if cfg else None, q, k, v, out,
                                    kp, vp, scales, table, ctx, starts, freq, qn, kn, None)


@pytest.mark.parametrize("kw", BAD_SHAPES, ids=str)
def test_append_bad_shapes_rejected(kw):
    assert append(shape(**kw), config()) == -2


def test_append_arguments_rejected():
    s, c = shape(), config()
    assert append(None, c) == -1 and append(s, None) == -1
    for name in ("q", "k", "v", "out", "kp", "vp", "scales", "table", "ctx", "starts", "freq"):
        assert append(s, c, **{name: None}) == -1, name
    for name in ("q", "k", "v", "out", "kp", "vp", "scales", "qn", "kn"):
        assert append(s, c, **{name: 24}) == -6, name
    for kw in (dict(rot_dim=24), dict(rot_dim=80), dict(rot_dim=-16), dict(interleaved=2), dict(reserved=1),
               dict(q_stride=504), dict(k_stride=120), dict(v_stride=132), dict(q_out_stride=0)):
        assert append(s, config(**kw)) == -6, kw
    assert append(s, config(eps=float("nan")), qn=16) == -6
    assert append(shape(num_tokens=0, max_q_len=0), None, q=None, scales=None) == 0


def decode(s, q=16, k=16, v=16, scales=16, table=16, ctx=16, ql=16, out=16, scale=0.125, ws=256, nbytes=1 << 40):
    return b.lib.ts_decode_attn_kv8(ctypes.byref(s) if s else None, q, k, v, scales, table, ctx, ql, out,
                                    ctypes.c_float(scale), ws, nbytes, None)


@pytest.mark.parametrize("kw", [dict(num_seqs=0), dict(num_q_heads=6, num_kv_heads=4), dict(head_dim=96),
                                dict(max_q_len=17), dict(num_q_heads=32, num_kv_heads=1, max_q_len=4),
                                dict(max_ctx_len=257), dict(num_pages=0), dict(num_workers=-1)], ids=str)
def test_decode_bad_shapes_rejected(kw):
    s = base_shape(**kw)
    assert b.lib.ts_decode_attn_kv8_workspace_size(ctypes.byref(s)) == 0 and decode(s) == -2


def test_decode_arguments_rejected():
    s = base_shape()
    need = b.decode_kv8_workspace_size(s)
    assert need > 0 and need % 256 == 0
    assert decode(None) == -1
    for name in ("q", "k", "v", "scales", "table", "ctx", "ql", "out", "ws"):
        assert decode(s, **{name: None}) == -1, name
    assert decode(s, nbytes=need - 1) == -3
    for kw in (dict(ws=128), dict(q=8), dict(k=24), dict(v=2), dict(scales=8), dict(out=8), dict(scale=float("nan"))):
        assert decode(s, **kw) == -6, kw
    for variant in (b.VARIANT_TEAM, b.VARIANT_VALU, 7):
        s = base_shape(head_dim=128)
        s.variant = variant
        assert decode(s) == -2 and b.lib.ts_decode_attn_kv8_workspace_size(ctypes.byref(s)) == 0


def test_decode_binding_refuses_other_tensors():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros(5, 2, 16, 64).to(torch.float8_e4m3fn)
    good = dict(q=torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16), k_pages=pages, v_pages=pages,
                kv_scales=torch.zeros(5, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu), page_table=i32(3, 2),
                ctx_lens=i32(3), q_lens=i32(3), out=torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16), scale=1.0)
    for name, bad in (("q", good["q"].float()), ("q", good["q"][:, :, ::2]), ("k_pages", pages.float()),
                      ("v_pages", pages[:4]), ("kv_scales", good["kv_scales"][:2]), ("page_table", i32(2, 2)),
                      ("ctx_lens", i32(4)), ("q_lens", i32(3, 1)), ("out", good["out"][:2])):
        with pytest.raises(ValueError, match=name):
            b.decode_attn_kv8(**{**good, name: bad})
    with pytest.raises(ValueError, match="CUDA"):
        b.decode_attn_kv8(**good)


def chunk(s, q=16, stride=512, k=16, v=16, scales=16, table=16, ctx=16, starts=16, out=16, out_stride=512, scale=0.125,
          ws=256, nbytes=1 << 40):
    return b.lib.ts_chunk_attn_kv8(ctypes.byref(s) if s else None, q, stride, k, v, scales, table, ctx, starts, out,
                                   out_stride, ctypes.c_float(scale), ws, nbytes, None)


@pytest.mark.parametrize("kw", BAD_SHAPES, ids=str)
def test_chunk_bad_shapes_rejected(kw):
    s = shape(**kw)
    assert b.lib.ts_chunk_attn_kv8_workspace_size(ctypes.byref(s)) == 0 and chunk(s) == -2


def test_chunk_arguments_rejected():
    s = shape()
    need = b.chunk_kv8_workspace_size(s)
    assert chunk(None) == -1
    for name in ("q", "k", "v", "scales", "table", "ctx", "starts", "out", "ws"):
        assert chunk(s, **{name: None}) == -1, name
    assert chunk(s, nbytes=need - 1) == -3
    for kw in (dict(ws=128), dict(q=8), dict(k=24), dict(v=2), dict(scales=4), dict(out=8), dict(stride=504),
               dict(out_stride=0), dict(scale=float("inf")), dict(out=16, q=16, out_stride=520)):
        assert chunk(s, **kw) == -6, kw
    assert chunk(shape(num_tokens=0, max_q_len=0), q=None, scales=None) == 0


def test_chunk_binding_refuses_other_tensors():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pages, rows = torch.zeros(5, 2, 16, 64).to(torch.float8_e4m3fn), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    good = dict(q=rows, k_pages=pages, v_pages=pages, kv_scales=torch.zeros(5, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu),
                page_table=i32(1, 2), ctx_lens=i32(1), q_starts=i32(2), out=rows.clone(), scale=1.0)
    for name, bad in (("q ", rows.float()), ("k_pages", pages.bfloat16()), ("v_pages", pages[:4]),
                      ("kv_scales", good["kv_scales"].view(torch.uint8)), ("page_table", i32(2)), ("ctx_lens", i32(2)),
                      ("q_starts", i32(3)), ("out", rows[:2])):
        with pytest.raises(ValueError, match=name):
            b.chunk_attn_kv8(**{**good, name.strip(): bad})
    with pytest.raises(ValueError, match="CUDA"):
        b.chunk_attn_kv8(**good)


def test_binding_refuses_other_types():
    bf, e4, e8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    rows = lambda h: torch.zeros(3, h, 64, dtype=bf)  # noqa: E731
    args = dict(q=rows(4), k=rows(2), v=rows(2), q_out=rows(4), k_pages=torch.zeros(5, 2, 16, 64).to(e4),
                v_pages=torch.zeros(5, 2, 16, 64).to(e4), kv_scales=torch.zeros(5, 2, 2, dtype=torch.uint8).view(e8),
                page_table=i32(1, 2), ctx_lens=i32(1), q_starts=i32(2), inv_freq=None)
    for name, bad in (("k_pages", torch.zeros(5, 2, 16, 64, dtype=bf)), ("v_pages", torch.zeros(5, 2, 16, 64, dtype=bf)),
                      ("kv_scales", torch.zeros(5, 2, 2, dtype=torch.uint8)), ("kv_scales", args["kv_scales"][:4]),
                      ("kv_scales", args["kv_scales"][..., :1])):
        with pytest.raises(ValueError, match=name):
            b.rope_append_kv8(**{**args, name: bad})
    with pytest.raises(ValueError, match="CUDA"):
        b.rope_append_kv8(**args)


def test_oracle_codes_are_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    mine, theirs = kv8.code_values(), codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mine, theirs, equal_nan=True)
    x = np.abs(mine[np.isfinite(mine)])
    grid = np.unique(x)
    for lo, hi in zip(grid[:-1], grid[1:]):
        assert hi - lo <= 2 * kv8.half_step(hi) and (hi - lo) / 2 == kv8.half_step(lo)


@pytest.mark.parametrize("amax,byte", [(448.0, 127), (448.0001, 128), (224.0, 126), (1.75, 119), (1.7500001, 120),
                                       (0.0, 27), (1e-30, 27), (3e38, 227), (2.0 ** -92, 27), (1.75 * 2.0 ** -91, 28)])
def test_oracle_power(amax, byte):
    assert kv8.power_byte(amax) == byte
    assert amax <= 448.0 * 2.0 ** (byte - 127) or byte == 227


def test_oracle_one_large_value_in_a_page():
    """What a page's one power costs: a value is off by at most half a step, 2^-4 of
    itself, but never less than 2^-10 of the power; below that it is lost."""
    rng = np.random.default_rng(3)
    heads, D = 1, 64
    k = rng.normal(size=(16, heads, D))
    k[5, 0, 7] = 448.0 * 2.0 ** 6
    codes, bytes_ = np.zeros((1, heads, 16, D), dtype=np.uint8), np.full((1, heads, 2), 127, dtype=np.uint8)
    _, want, _, after = kv8.append(k, k, k, codes, codes, bytes_, np.zeros((1, 1), dtype=int), [16], [0, 16], np.zeros(0))
    assert after[0, 0, 0] == 127 + 6
    grid = kv8.code_values()[:127]                                 # 0 .. 448, ascending
    size = np.abs(want[0, 0])
    held = np.sign(want[0, 0]) * grid[np.abs(size[..., None] - grid).argmin(-1)] * 2.0 ** 6
    x = k[:, 0]
    assert (np.abs(held - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * 2.0 ** 6)).all()
    assert (np.abs(held - x) <= kv8.half_step(size) * 2.0 ** 6).all()
    small = np.abs(x) < 2.0 ** -10 * 2.0 ** 6
    assert small.sum() > 20 and (held[small] == 0).all()           # lost whole
    middle = ~small & (np.abs(x) < 2.0 ** -6 * 2.0 ** 6)           # denormal codes
    assert (np.abs(held - x)[middle] > 2.0 ** -4 * np.abs(x)[middle]).any()


def test_every_call_hands_its_stream_and_tensors_to_the_device_check(monkeypatch):
    seen = []

    def check(*tensors, stream=None):
        seen.append((len(tensors), stream))
        raise ValueError("stop")

    monkeypatch.setattr(b, "_check_device", check)
    bf = lambda *s: torch.ones(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.ones(*s, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros(3, 2, 16, 64).to(torch.float8_e4m3fn)
    scales = torch.zeros(3, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    cache = (pages, pages, scales, i32(2, 2), i32(2))
    s = object()
    for call, n in ((lambda: b.chunk_attn_kv8(bf(5, 4, 64), *cache, i32(3), bf(5, 4, 64), 1.0, stream=s), 9),
                    (lambda: b.decode_attn_kv8(bf(2, 1, 4, 64), *cache, i32(2), bf(2, 1, 4, 64), 1.0, stream=s), 9),
                    (lambda: b.rope_append_kv8(bf(5, 4, 64), bf(5, 2, 64), bf(5, 2, 64), bf(5, 4, 64), *cache, i32(3), None,
                                               stream=s), 13),
                    (lambda: b.logit_rules(torch.ones(2, 8), torch.ones(2, 8), stream=s), 12)):
        with pytest.raises(ValueError, match="stop"):
            call()
        assert seen.pop() == (n, s)


@pytest.mark.parametrize("call, kind", [("decode_attn_kv8", "zeros"), ("chunk_attn_kv8", "empty")])
def test_own_workspaces_are_made_on_the_calls_stream(monkeypatch, call, kind):
    made = []
    monkeypatch.setattr(b, "_check_device", lambda *t, **kw: None)
    monkeypatch.setattr(b, "_stream_ptr", lambda s: 7)
    monkeypatch.setattr(b, "_own_workspace", lambda n, device, stream, zeros=False: made.append((stream, zeros)) or
                        torch.zeros(n, dtype=torch.uint8))
    monkeypatch.setattr(b, "check", lambda *a: None)
    monkeypatch.setattr(b.lib, "ts_" + call, lambda *a: 0)
    bf = lambda *s: torch.ones(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.ones(*s, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros(3, 2, 16, 64).to(torch.float8_e4m3fn)
    scales = torch.zeros(3, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    q, last = (bf(2, 1, 4, 64), i32(2)) if call.startswith("decode") else (bf(5, 4, 64), i32(3))
    stream = object()
    ws = getattr(b, call)(q, pages, pages, scales, i32(2, 2), i32(2), last, q.clone(), 1.0, stream=stream)
    assert made == [(stream, kind == "zeros")] and ws.numel() > 0


PARTITION = r"""
#include <cstdio>
#include <cstdlib>
#include "chunk_partition.h"
using namespace tsattn;
int main() {
    srand(11);
    for (int it = 0; it < 20000; it++) {
        ChunkSeq s;
        s.k8 = true;
        s.G = 1 + rand() % 16;
        s.TT = kTileRows / s.G;
        s.Q = 1 + rand() % (it % 2 ? 40 : 3000);
        s.P = rand() % (it % 3 ? 100 : 1000000);
        int64_t c = 0;
        for (int j = 0; j < s.tiles(); j++) {
            if (s.before(j) != c) { printf("before(%d): Q %d P %d G %d\n", j, s.Q, s.P, s.G); return 1; }
            const int rows = s.tokens(j) * s.G;
            c += (int64_t)s.cost(j) * (rows <= 16 ? 1 : rows <= 128 ? 2 : 3) + (rows <= 16 ? 8 : 20);
        }
        if (s.total() != c) return 2;
        if (c > places_bound(1, 1, s.Q, s.TT, (int64_t)s.P + s.Q, true)) return 3;
    }
    for (int G = 1; G <= 16; G++)
        if (places_bound(4096, 1024 / G, 1 << 22, kTileRows / G, 1ll << 30, true) >> 62) return 4;
    printf("ok\n");
    return 0;
}
"""


def test_partition_arithmetic(tmp_path):
    """Places of row tiles with the weights of this cache, against plain sums."""
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PARTITION)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2608_22788_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout + str(r.returncode)
