"""The largest work that chunk attention accepts is cut into ranges without
overflow: the limit on the workers, and the partition's arithmetic at it
against 128-bit integers."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_22788_amd import binding as b
from test_chunk import chunk, shape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGEST = dict(num_tokens=1 << 22, max_q_len=1 << 22, num_q_heads=1024, num_kv_heads=64, max_pages_per_seq=1 << 26,
               max_ctx_len=1 << 30, num_pages=1 << 31)


def size(**kw):
    return b.lib.ts_chunk_attn_workspace_size(ctypes.byref(shape(**kw)))


@pytest.mark.parametrize("seqs", [1, 4, 4096])
def test_workers_whose_ranges_would_overflow_are_refused(seqs):
    s = dict(LARGEST, num_seqs=seqs)
    assert size(**s, num_workers=1 << 16) == 0 and b"num_workers" in b.lib.ts_last_error()
    assert chunk(shape(**s, num_workers=1 << 16)) == -2
    assert size(**s) > 0                                  # the library's own choice fits
    # places of a row tile: two per 64 keys and 12 more; 16 tokens in each, all rows in every sequence
    places = seqs * 64 * (1 << 18) * (2 * (1 << 24) + 12)
    most = min((2 ** 63 - 1) // places, 1 << 16)
    assert size(**s, num_workers=most) > 0 and size(**s, num_workers=most + 1) == 0


def test_ordinary_calls_take_any_number_of_workers():
    for kw in (dict(num_seqs=4096, num_tokens=1 << 17, max_pages_per_seq=1 << 16, max_ctx_len=1 << 20),
               dict(num_seqs=1, num_tokens=1 << 20, max_pages_per_seq=1 << 17, max_ctx_len=1 << 21)):
        assert size(**kw, num_q_heads=32, num_kv_heads=8, head_dim=128, num_workers=1 << 16) > 0


PARTITION = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "chunk_partition.h"
using namespace tsattn;
typedef __int128 wide;
int main() {
    std::mt19937_64 rng(5);
    const auto upto = [&](uint64_t n) { return (int64_t)(rng() % (n + 1)); };
    // places_bound holds what any starts and lengths can ask for
    for (int it = 0; it < 20000; it++) {
        const int G = 1 + upto(15), TT = kTileRows / G, rows = 1 + upto(it % 2 ? 5000 : (1 << 22) - 1), Q = 1 + upto(rows - 1);
        const int64_t max_len = 16 * (1 + upto(it % 3 ? 1000 : (1 << 26) - 1)), L = upto(max_len);
        ChunkSeq s{Q, (int)(L > Q ? L - Q : 0), TT, G};
        if (s.total() > places_bound(1, 1, rows, TT, max_len)) { printf("bound: Q %d L %lld\n", Q, (long long)L); return 1; }
    }
    for (int G = 1; G <= 16; G++)
        if (places_bound(4096, 1024 / G, 1 << 22, kTileRows / G, 1ll << 30) >> 62) return 2;
    // range starts and the workers of places, up to the limit
    long n = 0;
    for (int it = 0; it < 200000; it++) {
        const int W = it % 4 == 0 ? 1 << 16 : 1 + (int)upto(it % 4 == 1 ? 255 : 65535);
        const int64_t most = INT64_MAX / W;
        const int64_t ptot = it % 8 == 7 ? most : 1 + upto((it % 3 ? most : (int64_t)1 << upto(40)) - 1);
        if (workers_bound(ptot) < W) return 3;
        const uint32_t inv = range_reciprocal(W);
        for (int k = 0; k < 4; k++) {
            const int w = k == 0 ? W : (int)upto(W);
            if ((wide)range_start(ptot, w, W, inv) != (wide)ptot * w / W) { printf("start %lld %d %d\n", (long long)ptot, w, W); return 4; }
            const int64_t x = k == 0 ? ptot - 1 : upto(ptot - 1);
            const int o = worker_of(ptot, x, W);
            if (o < 0 || o >= W || (wide)ptot * o / W > x || (wide)ptot * (o + 1) / W <= x) { printf("worker %lld %lld %d\n", (long long)ptot, (long long)x, W); return 5; }
            n++;
        }
    }
    printf("ok %ld\n", n);
    return 0;
}
"""


def test_partition_at_the_limit(tmp_path):
    src = tmp_path / "p.cpp"
    src.write_text(PARTITION)
    exe = tmp_path / "p"
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2608_22788_amd", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok"), (r.returncode, r.stdout)
