// chunk_partition.h -- how many KV tiles the row tiles of a chunk see: the
// integer arithmetic of chunk attention's work partition.  Plain C++, so that
// it is the same function on the host (tests) and in the kernels.
//
// A sequence of context length L with Q new tokens is cut into row tiles of TT
// tokens.  Row tile j (from 0) ends at token min(Q, (j + 1) TT) and sees the
// keys up to that token, so it takes ceil((P + min(Q, (j + 1) TT)) / 64) KV
// tiles of 64 keys, P = max(L - Q, 0) (tokens in front of the chunk).
//
// Workers share a line of places in equal ranges.  A KV tile has kTilePlaces
// places where the row tile keeps most wavefronts busy, one where up to half of
// its rows exist (that took about half as long), and belongs to the worker that
// holds its first place; kUnitPlaces more at the end of each row tile have no KV
// tile and stand for what starting and ending one costs, so that workers with
// many short row tiles get fewer KV tiles.
//
// With the cache held in 8 bits a place is 0.7 us: a KV tile takes that long where a
// row tile has up to kFewRows rows (6 us for starting and ending one), 1.2 us up to
// half of the rows, 2.3 us with more (14 us).
#pragma once

#include <stdint.h>

#include "partition.h"

namespace tsattn {

constexpr int kKeyTile = 64;   // keys per KV tile
constexpr int kTileRows = 256; // rows (tokens x query heads of a KV head) per row tile
constexpr int kTilePlaces = 2, kUnitPlaces = 12;
constexpr int kFewRows = 16;
constexpr int kTilePlaces8 = 3, kUnitPlaces8 = 20, kFewUnitPlaces8 = 8;

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
    int G;      // query heads per KV head
    bool k8 = false;   // the cache is held in 8 bits
    TS_HOST_DEVICE int tiles() const { return (int)(((int64_t)Q + TT - 1) / TT); }
    // tokens of row tile j
    TS_HOST_DEVICE int tokens(int j) const {
        const int left = Q - j * TT;
        return left < TT ? left : TT;
    }
    // KV tiles of row tile j
    TS_HOST_DEVICE int cost(int j) const { return (P + j * TT + tokens(j) + kKeyTile - 1) / kKeyTile; }
    // places of one of them
    TS_HOST_DEVICE int weight(int j) const {
        const int rows = tokens(j) * G;
        if (k8)
            return rows > kTileRows / 2 ? kTilePlaces8 : rows > kFewRows ? 2 : 1;
        return rows > kTileRows / 2 ? kTilePlaces : 1;
    }
    // and behind them
    TS_HOST_DEVICE int behind(int j) const {
        return !k8 ? kUnitPlaces : tokens(j) * G > kFewRows ? kUnitPlaces8 : kFewUnitPlaces8;
    }
    // places of row tiles 0 .. j - 1
    TS_HOST_DEVICE int64_t before(int j) const {
        const int full = Q / TT, n = j < full ? j : full;
        int64_t c = 0;
        if (n > 0)
            c = weight(0) * floor_sum64((uint32_t)n, (uint32_t)TT, (uint64_t)P + TT + kKeyTile - 1) + (int64_t)n * behind(0);
        if (j > full)
            c += (int64_t)weight(full) * cost(full) + behind(full);
        return c;
    }
    TS_HOST_DEVICE int64_t total() const { return before(tiles()); }
};

// Places of a call from above, whatever its arrays hold (starts out of order can
// give every sequence all the rows); below 2^62 for every accepted shape.  The
// cut into W ranges multiplies places by W in 64 bits.
inline int64_t places_bound(int seqs, int kv_heads, int rows, int TT, int64_t max_len, bool k8 = false) {
    const int64_t tiles = ((int64_t)rows + TT - 1) / TT;
    const int64_t keys = max_len > rows ? max_len : rows;
    return (int64_t)seqs * kv_heads * tiles *
           ((k8 ? kTilePlaces8 : kTilePlaces) * ((keys + kKeyTile - 1) / kKeyTile) + (k8 ? kUnitPlaces8 : kUnitPlaces));
}
inline int64_t workers_bound(int64_t places) { return INT64_MAX / (places > 0 ? places : 1); }

// First KV tile at or behind place `off` of a row tile.
TS_HOST_DEVICE int tile_at(int64_t off, int weight) { return (int)((off + weight - 1) / weight); }

}  // namespace tsattn
