"""The operators on packed rows without a GPU: their refusals before any HIP
call, the work partition's arithmetic against plain loops, and the float64
oracle against hand-worked cases."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import chunk as orc
from paper_2608_22788_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def shape(**kw):
    d = dict(num_seqs=4, num_tokens=40, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_q_len=30,
             max_pages_per_seq=16, max_ctx_len=256, num_workers=0, num_pages=64)
    d.update(kw)
    return b.ChunkShape(*(d[f] for f, _ in b.ChunkShape._fields_))


def chunk(s, q=16, stride=512, k=16, v=16, table=16, ctx=16, starts=16, out=16, out_stride=512, scale=0.125, ws=256,
          nbytes=1 << 40):
    return b.lib.ts_chunk_attn(ctypes.byref(s) if s else None, q, stride, k, v, table, ctx, starts, out, out_stride,
                               ctypes.c_float(scale), ws, nbytes, None)


def rope(s, cfg, q=16, k=16, v=16, out=16, kp=16, vp=16, table=16, ctx=16, starts=16, freq=16, qn=None, kn=None):
    return b.lib.ts_rope_append(ctypes.byref(s) if s else None, ctypes.byref(cfg) if cfg else None, q, k, v, out, kp,
                                vp, table, ctx, starts, freq, qn, kn, None)


def config(**kw):
    d = dict(rot_dim=64, interleaved=0, eps=1e-6, reserved=0, q_stride=512, k_stride=128, v_stride=128,
             q_out_stride=512)
    d.update(kw)
    return b.RopeConfig(*(d[f] for f, _ in b.RopeConfig._fields_))


BAD_SHAPES = [dict(num_seqs=0), dict(num_seqs=4097), dict(num_tokens=-1), dict(num_tokens=(1 << 22) + 1),
              dict(num_q_heads=6, num_kv_heads=4), dict(num_kv_heads=0), dict(num_q_heads=34), dict(num_q_heads=0),
              dict(num_q_heads=2048, num_kv_heads=1024), dict(head_dim=96), dict(head_dim=256), dict(page_size=32),
              dict(max_q_len=-1), dict(max_q_len=41), dict(max_pages_per_seq=0), dict(max_pages_per_seq=(1 << 26) + 1),
              dict(max_ctx_len=0), dict(max_ctx_len=257), dict(num_pages=0), dict(num_workers=-1),
              dict(num_workers=1 << 17)]


@pytest.mark.parametrize("kw", BAD_SHAPES, ids=str)
def test_bad_shapes_rejected(kw):
    s = shape(**kw)
    assert b.lib.ts_chunk_attn_workspace_size(ctypes.byref(s)) == 0
    assert b.lib.ts_last_error()
    assert chunk(s) == -2
    assert rope(s, config()) == -2


def test_chunk_arguments_rejected():
    s = shape()
    need = b.chunk_workspace_size(s)
    assert need > 0 and need % 256 == 0
    assert chunk(None) == -1
    for name in ("q", "k", "v", "table", "ctx", "starts", "out", "ws"):
        assert chunk(s, **{name: None}) == -1, name
    assert chunk(s, nbytes=need - 1) == -3
    for kw in (dict(ws=128), dict(q=8), dict(k=24), dict(v=2), dict(out=8), dict(stride=504), dict(stride=516),
               dict(out_stride=0), dict(out_stride=-512), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert chunk(s, **kw) == -6, kw


def test_rope_arguments_rejected():
    s = shape()
    assert rope(None, config()) == -1
    assert rope(s, None) == -1
    for name in ("q", "k", "v", "out", "kp", "vp", "table", "ctx", "starts", "freq"):
        assert rope(s, config(), **{name: None}) == -1, name
    for kw in (dict(rot_dim=-16), dict(rot_dim=8), dict(rot_dim=80), dict(interleaved=2), dict(q_stride=504),
               dict(k_stride=120), dict(v_stride=132), dict(q_out_stride=0), dict(reserved=1)):
        assert rope(s, config(**kw)) == -6, kw
    assert rope(s, config(q_out_stride=520)) == -6                       # in place with another stride
    for eps in (-1.0, float("nan"), float("inf")):
        assert rope(s, config(eps=eps), qn=16) == -6
    for kw in (dict(q=8), dict(k=8), dict(v=8), dict(out=8), dict(kp=8), dict(vp=8), dict(qn=8), dict(kn=8)):
        assert rope(s, config(), **kw) == -6, kw


def test_no_rows_is_no_work():
    s = shape(num_tokens=0, max_q_len=0)
    assert chunk(s, q=None, out=None) == 0
    assert rope(s, config(), q=None, k=None, v=None, out=None) == 0


PARTITION = r"""
#include <cstdio>
#include <cstdlib>
#include "chunk_partition.h"
using namespace tsattn;
int main() {
    srand(7);
    long n = 0;
    for (int it = 0; it < 20000; it++) {
        ChunkSeq s;
        s.G = 1 + rand() % 16;
        s.TT = kTileRows / s.G;
        s.Q = 1 + rand() % (it % 2 ? 40 : 3000);
        s.P = rand() % (it % 3 ? 100 : 1000000);
        int64_t c = 0;
        int row = 0;
        for (int j = 0; j < s.tiles(); j++) {
            if (s.before(j) != c) { printf("before(%d): Q %d P %d G %d\n", j, s.Q, s.P, s.G); return 1; }
            const int last = row + s.TT < s.Q ? row + s.TT : s.Q;   // tokens up to the tile's last
            int tiles = 0;
            if (s.P < 5000) {
                for (long t = 0; t < (long)s.P + last; t += 64) tiles++;
                if (tiles != s.cost(j)) { printf("cost(%d): Q %d P %d G %d\n", j, s.Q, s.P, s.G); return 1; }
            }
            if (s.tokens(j) != last - row || s.weight(j) != ((last - row) * s.G > 128 ? 2 : 1)) return 2;
            c += (int64_t)s.cost(j) * s.weight(j) + kUnitPlaces;
            row = last;
            n++;
        }
        if (row != s.Q || s.total() != c) { printf("total: Q %d P %d G %d\n", s.Q, s.P, s.G); return 1; }
        // a boundary anywhere in a row tile gives each KV tile to one side
        const int w = s.weight(0), k = s.cost(0);
        for (int off = 0; off <= k * w && off < 200; off++) {
            int mine = 0;
            for (int j = 0; j < k && j < 200; j++) mine += j * w < off;
            if (tile_at(off, w) != mine) return 3;
        }
    }
    ChunkSeq s{1 << 22, 1 << 30, 16, 16};   // the largest chunk behind the longest context
    int64_t c = 0;
    for (int j = 0; j < s.tiles(); j++) c += (int64_t)s.cost(j) * s.weight(j) + kUnitPlaces;
    if (c != s.total()) return 1;
    printf("ok %ld\n", n);
    return 0;
}
"""


def test_partition_arithmetic(tmp_path):
    src = tmp_path / "p.cpp"
    src.write_text(PARTITION)
    exe = tmp_path / "p"
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2608_22788_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout


# ---- the oracle ---------------------------------------------------------------------

def test_oracle_attention_hand_case():
    """Two keys with equal scores: the first row sees one, the second their mean."""
    D = 4
    kp, vp = np.zeros((1, 1, 16, D)), np.zeros((1, 1, 16, D))
    vp[0, 0, 0], vp[0, 0, 1] = 1.0, 3.0
    vp[0, 0, 2:] = np.nan
    out, mag = orc.chunk_attention(np.ones((3, 2, D)), kp, vp, np.zeros((1, 1), int), [2], [0, 2], 0.5)
    assert np.allclose(out[0], 1.0) and np.allclose(out[1], 2.0) and np.isnan(out[2]).all()
    assert np.allclose(mag[:2], out[:2])


def test_oracle_attention_matches_the_library_oracle():
    """Against the C oracle of decode attention on a padded batch."""
    import oracle
    rng = np.random.default_rng(0)
    B, Qm, Hq, Hkv, D, npg = 2, 3, 4, 2, 64, 6
    bf = lambda x: (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731
    val = lambda u: (u.astype(np.uint32) << 16).view(np.float32).astype(np.float64)  # noqa: E731
    q, kp, vp = (bf(rng.normal(size=s)) for s in ((B, Qm, Hq, D), (npg, Hkv, 16, D), (npg, Hkv, 16, D)))
    table, ctx, ql = np.array([[3, 1, 0], [5, 2, 4]], np.int32), np.array([37, 40], np.int32), np.array([3, 2], np.int32)
    oracle.build()
    want = oracle.load().attention(q, kp, vp, table, ctx, ql, 0.125)
    packed = np.concatenate([val(q[0]), val(q[1, :2])])
    got, _ = orc.chunk_attention(packed, val(kp), val(vp), table, ctx, [0, 3, 5], 0.125)
    assert np.allclose(got[:3], want[0], atol=1e-12) and np.allclose(got[3:], want[1, :2], atol=1e-12)


def test_oracle_rope_turns_pairs_by_the_position():
    f = np.array([1.0, 0.5])
    q = np.zeros((1, 1, 6))
    q[0, 0, :4] = [1.0, 0.0, 0.0, 0.0]
    q[0, 0, 4:] = 7.0
    pages = np.zeros((1, 1, 16, 6))
    out, kp, _ = orc.rope_append(q, q, q, pages, pages, np.zeros((1, 1), int), [3], [0, 1], f)
    assert np.allclose(out[0, 0], [np.cos(2), 0, np.sin(2), 0, 7, 7]) and np.allclose(kp[0, 0, 2], out[0, 0])
    out, _, vp = orc.rope_append(q, q, q, pages, pages, np.zeros((1, 1), int), [3], [0, 1], f, interleaved=True)
    assert np.allclose(out[0, 0], [np.cos(2), np.sin(2), 0, 0, 7, 7]) and np.allclose(vp[0, 0, 2], q[0, 0])
    out, _, _ = orc.rope_append(q, q, q, pages, pages, np.zeros((1, 1), int), [3], [0, 1], f[:0], np.full(6, 2.0), eps=0.0)
    assert np.allclose(out[0, 0, 4], 14.0 / np.sqrt(99.0 / 6.0))
