// chunk_partition.h -- how many KV tiles the row tiles of a chunk see: the
// integer arithmetic of chunk attention's work partition.  Plain C++, so that
// it is the same function on the host (tests) and in the kernels.
//
// A sequence of context length L with Q new tokens is cut into row tiles of TT
// tokens.  Row tile j (from 0) ends at token min(Q, (j + 1) TT) and sees the
// keys up to that token, so it takes ceil((P + min(Q, (j + 1) TT)) / 64) KV
// tiles of 64 keys, P = max(L - Q, 0) (tokens in front of the chunk).  Its
// share of the line of work is kUnitTiles longer: behind its KV tiles lie that
// many places without any, so that workers with many short row tiles get
// fewer KV tiles.
#pragma once

#include <stdint.h>

#include "partition.h"

namespace tsattn {

constexpr int kKeyTile = 64;   // keys per KV tile
constexpr int kUnitTiles = 6;  // what starting and ending a row tile costs, in KV tiles

// sum over i = 0 .. n - 1 of floor((a i + b) / 64), for n <= 2^23, a <= 256:
// whole multiples of 64 leave a and b, then the roles of the axes are swapped
// until no lattice point is left (as in Euclid's algorithm).
TS_HOST_DEVICE int64_t floor_sum64(uint32_t n, uint32_t a, uint64_t b) {
    int64_t sum = (int64_t)n * (int64_t)(b / kKeyTile) +
                  (int64_t)(a / kKeyTile) * ((int64_t)n * ((int64_t)n - 1) / 2);
    uint32_t m = kKeyTile, r = (uint32_t)(b % kKeyTile);
    a %= kKeyTile;
    for (;;) {   // a < m, r < m
        const uint32_t y = a * n + r;   // below 2^6 (2^23 + 1)
        if (y < m)
            return sum;
        n = y / m;
        r = y - n * m;
        const uint32_t t = m;
        m = a;
        a = t;
        // whole multiples of the new modulus
        const uint32_t qa = a / m, qr = r / m;
        sum += (int64_t)qa * ((int64_t)n * ((int64_t)n - 1) / 2) + (int64_t)qr * n;
        a -= qa * m;
        r -= qr * m;
    }
}

struct ChunkSeq {
    int Q;      // new tokens
    int P;      // tokens in front of them
    int TT;     // tokens per row tile
    TS_HOST_DEVICE int tiles() const { return (int)(((int64_t)Q + TT - 1) / TT); }
    // KV tiles of row tile j
    TS_HOST_DEVICE int keys_end(int j) const {
        const int64_t e = (int64_t)(j + 1) * TT;
        return P + (int)(e < Q ? e : Q);
    }
    TS_HOST_DEVICE int cost(int j) const { return (keys_end(j) + kKeyTile - 1) / kKeyTile; }
    // places of row tiles 0 .. j - 1
    TS_HOST_DEVICE int64_t before(int j) const {
        const int full = Q / TT, n = j < full ? j : full;
        int64_t c = floor_sum64((uint32_t)n, (uint32_t)TT, (uint64_t)P + TT + kKeyTile - 1);
        if (j > full)
            c += cost(full);
        return c + (int64_t)j * kUnitTiles;
    }
    TS_HOST_DEVICE int64_t total() const { return before(tiles()); }
};

}  // namespace tsattn
