// chunk_attn.hip -- attention of chunks of new tokens over the paged cache.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attn_common.h"
#include "chunk_common.h"
#include "chunk_partition.h"
#include "ts_attn.h"
#include "ts_internal.h"

namespace tsattn {

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kRowBlock = 32;      // rows of a matrix-core tile
constexpr int kChunkWaves = 4;
constexpr int kTileRows = kChunkWaves * kRowBlock;
constexpr float kTiny = 1.17549435e-38f;   // the smallest normal float32
constexpr int kTilePages = kKeyTile / kPage;

struct ChunkParams {
    const uint16_t *q;          // [num_tokens][Hq][D], rows of q_stride elements
    const uint16_t *k_pages;    // [num_pages][Hkv][16][D]
    const uint16_t *v_pages;
    const int32_t *page_table;  // [B][max_pages]
    const int32_t *ctx_lens;    // [B]
    const int32_t *q_starts;    // [B + 1]
    uint16_t *out;
    float *ws_o;                // [2W][kTileRows][D] partial outputs, normalised
    float *ws_lse;              // [2W][kTileRows] log2-sum-exp
    int64_t q_stride, out_stride, num_pages;
    int B, Hq, Hkv, G, max_pages, num_tokens;
    int TT;                     // tokens per row tile
    int W;                      // workers
    uint32_t range_inv;
    float scale_log2;           // |scale| * log2(e)
    uint32_t q_sign;            // sign bits to flip in a pair of q values
};

// Sequence b: its first packed row, new tokens and tokens in front of them.
// Row and length limits keep every access in bounds whatever the arrays hold.
struct SeqInfo {
    int row0, L;
    ChunkSeq c;
};
__device__ __forceinline__ SeqInfo seq_info(const ChunkParams &p, int b) {
    SeqInfo s;
    const int a = min(max(ld_meta(p.q_starts, b), 0), p.num_tokens);
    const int e = min(max(ld_meta(p.q_starts, b + 1), 0), p.num_tokens);
    s.row0 = a;
    s.c.Q = max(e - a, 0);
    s.L = (int)min((int64_t)max(ld_meta(p.ctx_lens, b), 0), (int64_t)p.max_pages * kPage);
    s.c.P = max(s.L - s.c.Q, 0);
    s.c.TT = p.TT;
    return s;
}

// Exclusive prefix over the sequences of one head's KV tiles, in s_pre[0..B].
__device__ inline void tile_prefix(const ChunkParams &p, uint64_t *s_pre) {
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x;
        uint64_t base = 0;
        for (int b0 = 0; b0 < p.B; b0 += kWave) {
            const int b = b0 + lane;
            uint64_t n = 0;
            if (b < p.B) {
                const SeqInfo s = seq_info(p, b);
                n = s.c.Q > 0 ? (uint64_t)s.c.total() : 0;
            }
            const uint64_t incl = wave_incl_scan(n);
            if (b < p.B)
                s_pre[b] = base + incl - n;
            base += __shfl(incl, kWave - 1, kWave);
        }
        if (lane == 0)
            s_pre[p.B] = base;
    }
    __syncthreads();
}

struct Piece {
    int b, g, m;       // sequence, KV head, row tile
    int j0, j1;        // KV tiles [j0, j1) of it
    int n;             // KV tiles of the whole unit
    bool whole;
    int64_t us;        // global index of the unit's first KV tile
    int64_t next;
};

// The unit that holds global tile x, and the part of it in [x, range_end).
// Units are laid out sequence by sequence, head by head, row tile by row tile.
__device__ inline Piece locate_tile(const ChunkParams &p, const uint64_t *s_pre, int64_t x, int64_t range_end) {
    const int lane = threadIdx.x & (kWave - 1);
    Piece r;
    // the last sequence that starts at or before x
    int lo = 0, n = p.B;
    if (p.B > kWave) {
        const int step = (p.B + kWave - 1) / kWave;
        const int at = lane * step;
        lo = step * (__popcll(__ballot(at < p.B && (int64_t)s_pre[min(at, p.B)] * p.Hkv <= x)) - 1);
        n = min(step, p.B - lo);
    }
    r.b = first_lane_int(lo + __popcll(__ballot(lane < n && (int64_t)s_pre[min(lo + lane, p.B)] * p.Hkv <= x)) - 1);
    const int64_t pre = first_lane_int64((int64_t)s_pre[r.b]);
    const int64_t per_head = first_lane_int64((int64_t)s_pre[r.b + 1]) - pre;
    const int64_t off = x - pre * p.Hkv;
    r.g = first_lane_int((int)(off / per_head));
    const int64_t in_head = off - r.g * per_head;
    const ChunkSeq c = seq_info(p, r.b).c;
    // the last row tile that starts at or before in_head
    int m = 0, span = c.tiles();
    while (span > 1) {
        const int step = (span + kWave - 1) / kWave;
        const int at = m + lane * step;
        const bool le = lane * step < span && c.before(at) <= in_head;
        const int k = __popcll(__ballot(le)) - 1;
        const int skip = max(k, 0) * step;
        m += skip;
        span = min(step, span - skip);
    }
    r.m = first_lane_int(m);
    const int64_t start = c.before(r.m);
    r.n = c.cost(r.m);
    r.us = x - in_head + start;
    r.j0 = first_lane_int((int)(in_head - start));
    const int64_t unit_end = r.us + r.n;
    r.next = unit_end < range_end ? unit_end : range_end;
    r.j1 = first_lane_int((int)(r.next - r.us));
    r.whole = r.j0 == 0 && r.j1 == r.n;
    return r;
}

__device__ __forceinline__ float max_both_halves(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float sum_both_halves(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D>
struct Chunk {
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kPieces = kRowBytes / 16;         // 16-byte pieces of a row
    static constexpr int kVPitch = kRowBytes + 32;
    static constexpr int kKBytes = kKeyTile * kRowBytes;
    static constexpr int kVBytes = kKeyTile * kVPitch;
    static constexpr int kStage = kKBytes + kVBytes;
    static constexpr int kLds = 2 * kStage;
    static constexpr int kLoads = kPage * kRowBytes / (16 * kWave);   // loads of a wave per page block
    static constexpr int kKSteps = D / 16;
    static constexpr int kDTiles = D / 32;

    struct Stage {
        u32x4_t k[kLoads], v[kLoads];
    };

    // Wave w loads page w of KV tile j: rows at or past `L` and pages outside
    // the pool read as zeros (buffer bounds), without a memory access.
    __device__ __forceinline__ static void load_tile(const ChunkParams &p, const int32_t *pt, int g, int j, int L, int wave, int lane,
                                     Stage &s) {
        const int page = j * kTilePages + wave;
        const int rows = min(max(L - page * kPage, 0), kPage);
        const int pid = ld_meta(pt, rows > 0 ? page : 0);
        const bool ok = rows > 0 && pid >= 0 && pid < p.num_pages;
        const size_t base = ((size_t)(ok ? pid : 0) * p.Hkv + g) * (size_t)(kPage * D);
        const int bytes = ok ? rows * kRowBytes : 0;
        const block_rsrc_t rk = block_rsrc(p.k_pages + base, bytes);
        const block_rsrc_t rv = block_rsrc(p.v_pages + base, bytes);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            s.k[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, 16 * (i * kWave + lane), 0, 0);
            s.v[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, 16 * (i * kWave + lane), 0, 0);
        }
    }

    __device__ __forceinline__ static int k_addr(int key, int piece) {
        return key * kRowBytes + ((piece ^ (key & (kPieces - 1))) << 4);
    }

    // `clean`: infinite and NaN values are staged as zero; returns whether there were any.
    __device__ __forceinline__ static bool store_tile(char *stage, int wave, int lane, Stage &s, bool clean) {
        bool odd = false;
        if (clean)
#pragma unroll
            for (int i = 0; i < kLoads; i++)
                odd |= clear_odd(s.v[i]);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int at = i * kWave + lane;
            const int key = kPage * wave + at / kPieces, piece = at % kPieces;
            *reinterpret_cast<u32x4_t *>(stage + k_addr(key, piece)) = s.k[i];
            *reinterpret_cast<u32x4_t *>(stage + kKBytes + key * kVPitch + 16 * piece) = s.v[i];
        }
        return odd;
    }

    struct State {
        u32x4_t qf[kKSteps];
        f32x16_t o[kDTiles];
        float m_ref, l;
        int lim;      // keys that this lane's row sees
    };

    __device__ __forceinline__ static bf16x8_t v_frag(const char *v, int dt, int step, int lane) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
        const int h = lane >> 5, i = lane & 15;
        const char *at = v + (16 * step + 4 * h + (i >> 2)) * kVPitch + 2 * (32 * dt + 16 * ((lane >> 4) & 1) + 4 * (i & 3));
        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(__attribute__((address_space(3))) const char *)at);
        const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4 *)(__attribute__((address_space(3))) const char *)(at + 8 * kVPitch));
        s16x4_t ab[2] = {a, b};
        return __builtin_bit_cast(bf16x8_t, ab);
    }

    // Infinite and NaN values.  Where a row does not see a key, the key's zero
    // weight would still make NaN of such a value in the matrix product.  So in
    // the tiles that some row of the unit does not see whole (the last one to
    // three) they are replaced by zero when the tile is staged, and put back
    // afterwards for the rows that see them, whose result is infinite or NaN
    // whatever the weight.
    static __device__ __forceinline__ bool clear_odd(u32x4_t &v) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const bool lo = (v[i] & 0x7f80u) == 0x7f80u, hi = (v[i] & 0x7f800000u) == 0x7f800000u;
            odd |= lo || hi;
            v[i] = lo ? v[i] & 0xffff0000u : v[i];
            v[i] = hi ? v[i] & 0x0000ffffu : v[i];
        }
        return odd;
    }

    static __device__ __forceinline__ float put_back(float o, uint32_t x) {   // x: a bf16 value in the high half
        return (x & 0x7f800000u) == 0x7f800000u ? o + __uint_as_float(x) : o;
    }

    __device__ __forceinline__ static void add_odd(const ChunkParams &p, State &st, const int32_t *pt, int g, int t0, int t1, int h) {
#pragma unroll 1
        for (int t = t0; t < t1; t++) {
            const int pid = ld_meta(pt, t / kPage);
            if (pid < 0 || pid >= p.num_pages)
                continue;
            const uint16_t *row = p.v_pages + (((size_t)pid * p.Hkv + g) * kPage + t % kPage) * D + 4 * h;
            if (t >= st.lim)
                continue;
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(row + 32 * dt + 8 * e);
                    st.o[dt][4 * e] = put_back(st.o[dt][4 * e], x.x << 16);
                    st.o[dt][4 * e + 1] = put_back(st.o[dt][4 * e + 1], x.x & 0xffff0000u);
                    st.o[dt][4 * e + 2] = put_back(st.o[dt][4 * e + 2], x.y << 16);
                    st.o[dt][4 * e + 3] = put_back(st.o[dt][4 * e + 3], x.y & 0xffff0000u);
                }
        }
    }

    __device__ __forceinline__ static void tile_step(const ChunkParams &p, State &st, const char *stage, int j, bool masked, int lane) {
        const int n = lane & 31, h = lane >> 5;
        f32x16_t s[2];
#pragma unroll
        for (int kt = 0; kt < 2; kt++) {
#pragma unroll
            for (int e = 0; e < 16; e++)
                s[kt][e] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < kKSteps; ks++) {
                const u32x4_t kf = *reinterpret_cast<const u32x4_t *>(stage + k_addr(32 * kt + n, 2 * ks + h));
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf),
                                                                __builtin_bit_cast(bf16x8_t, st.qf[ks]), s[kt], 0, 0, 0);
            }
        }
        const int room = st.lim - j * kKeyTile - 4 * h;   // key offset 8 (e / 4) + e % 4 + 32 kt is seen if below
        if (masked) {
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    s[kt][e] = 32 * kt + 8 * (e / 4) + e % 4 < room ? s[kt][e] : -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e++)
                mx = fmaxf(mx, s[kt][e]);
        mx *= p.scale_log2;
        if (__any(mx > st.m_ref + kRescaleSlack)) {
            mx = max_both_halves(mx);
            const bool up = mx > st.m_ref + kRescaleSlack;
            // (never zero, so that an infinite sum stays infinite)
            const float alpha = up ? fmaxf(fast_exp2(st.m_ref - mx), kTiny) : 1.0f;
            st.m_ref = up ? mx : st.m_ref;
            st.l *= alpha;
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    st.o[dt][e] *= alpha;
        }
        u32x4_t pf[4];   // four steps of 16 keys
#pragma unroll
        for (int kt = 0; kt < 2; kt++) {
#pragma unroll
            for (int e = 0; e < 16; e++) {
                float x = fast_exp2(__builtin_fmaf(s[kt][e], p.scale_log2, -st.m_ref));
                if (masked)
                    x = 32 * kt + 8 * (e / 4) + e % 4 < room ? x : 0.0f;
                st.l += x;
                s[kt][e] = x;
            }
#pragma unroll
            for (int e = 0; e < 8; e++)
                pf[2 * kt + e / 4][e % 4] = pack_bf16x2(s[kt][2 * e], s[kt][2 * e + 1]);
        }
        const char *v = stage + kKBytes;
#pragma unroll
        for (int step = 0; step < 4; step++)
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
                st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(v, dt, step, lane),
                                                                   __builtin_bit_cast(bf16x8_t, pf[step]), st.o[dt], 0, 0, 0);
    }

    __device__ __forceinline__ static void piece(const ChunkParams &p, const Piece &pc, int slot, char *lds) {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = first_lane_int(threadIdx.x / kWave);
        const int h = lane >> 5;
        const SeqInfo sq = seq_info(p, pc.b);
        const int32_t *pt = p.page_table + (size_t)pc.b * p.max_pages;
        const int r = wave * kRowBlock + (lane & 31);
        const int token = pc.m * p.TT + r / p.G;
        const bool row_ok = r < p.TT * p.G && token < sq.c.Q;
        const int head = pc.g * p.G + r % p.G;
        State st;
        st.lim = row_ok ? sq.L - sq.c.Q + token + 1 : 0;
        st.m_ref = -INFINITY;
        st.l = 0.0f;
        const uint16_t *qr = p.q + (int64_t)(sq.row0 + (row_ok ? token : 0)) * p.q_stride + (int64_t)(row_ok ? head : 0) * D + 8 * h;
#pragma unroll
        for (int ks = 0; ks < kKSteps; ks++) {
            st.qf[ks] = row_ok ? *reinterpret_cast<const u32x4_t *>(qr + 16 * ks) : u32x4_t{0u, 0u, 0u, 0u};
            st.qf[ks] ^= p.q_sign;
        }
#pragma unroll
        for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
            for (int e = 0; e < 16; e++)
                st.o[dt][e] = 0.0f;
        // rows go by token and the valid ones come first, so the wave's first
        // row sees the fewest keys; what rows without a token hold is not used
        const int lo_lim = __builtin_amdgcn_readlane(st.lim, 0);
        int hi_lim = st.lim;
        for (int d = 16; d; d >>= 1)
            hi_lim = max(hi_lim, __shfl_xor(hi_lim, d, kWave));
        hi_lim = first_lane_int(hi_lim);

        Stage sg;
        load_tile(p, pt, pc.g, pc.j0, sq.L, wave, lane, sg);
        // the first row of the unit sees the fewest keys
        const int all_lim = sq.L - sq.c.Q + pc.m * p.TT + 1;
        bool odd = store_tile(lds, wave, lane, sg, (pc.j0 + 1) * kKeyTile > all_lim);
        lds_barrier();
        for (int j = pc.j0; j < pc.j1; j++) {
            const int cur = (j - pc.j0) & 1;
            if (j + 1 < pc.j1)
                load_tile(p, pt, pc.g, j + 1, sq.L, wave, lane, sg);
            if (j * kKeyTile < hi_lim)
                tile_step(p, st, lds + cur * kStage, j, (j + 1) * kKeyTile > lo_lim, lane);
            if (j + 1 < pc.j1)
                odd |= store_tile(lds + (cur ^ 1) * kStage, wave, lane, sg, (j + 2) * kKeyTile > all_lim);
            lds_barrier();
        }
        if (pc.j1 * kKeyTile > all_lim) {   // the same for every wavefront
            int *flags = reinterpret_cast<int *>(lds);
            const bool mine = __any(odd);
            if (lane == 0)
                flags[wave] = mine;
            lds_barrier();
            bool any = false;
#pragma unroll
            for (int i = 0; i < kChunkWaves; i++)
                any |= flags[i] != 0;
            lds_barrier();
            if (any)
                add_odd(p, st, pt, pc.g, max(pc.j0, max(all_lim, 0) / kKeyTile) * kKeyTile, min(pc.j1 * kKeyTile, sq.L), h);
        }
        if (!row_ok)
            return;
        const float l = sum_both_halves(st.l);
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // NaN stays
        if (pc.whole) {
            uint16_t *dst = p.out + (int64_t)(sq.row0 + token) * p.out_stride + (int64_t)head * D + 4 * h;
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    *reinterpret_cast<uint2 *>(dst + 32 * dt + 8 * e) =
                        make_uint2(pack_bf16x2(st.o[dt][4 * e] * inv, st.o[dt][4 * e + 1] * inv),
                                   pack_bf16x2(st.o[dt][4 * e + 2] * inv, st.o[dt][4 * e + 3] * inv));
        } else {
            const int64_t row = (int64_t)slot * kTileRows + r;
            float *dst = p.ws_o + row * D + 4 * h;
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    f32x4_t x;
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        x[i] = st.o[dt][4 * e + i] * inv;
                    *reinterpret_cast<f32x4_t *>(dst + 32 * dt + 8 * e) = x;
                }
            if (h == 0)
                p.ws_lse[row] = l == 0.0f ? -INFINITY : st.m_ref + __log2f(l);
        }
    }
};

template <int D>
__global__ __launch_bounds__(kChunkWaves * kWave, 2) void chunk_attn_kernel(ChunkParams p) {
    extern __shared__ uint64_t s_tiles[];
    char *lds = reinterpret_cast<char *>(s_tiles) + (((p.B + 1) * 8 + 127) & ~127);
    tile_prefix(p, s_tiles);
    const int64_t ptot = (int64_t)s_tiles[p.B] * p.Hkv;
    const int w = xcd_worker(blockIdx.x, p.W);
    const int64_t begin = first_lane_int64(range_start(ptot, w, p.W, p.range_inv));
    const int64_t end = first_lane_int64(range_start(ptot, w + 1, p.W, p.range_inv));
    for (int64_t x = begin; x < end;) {
        const Piece pc = locate_tile(p, s_tiles, x, end);
        Chunk<D>::piece(p, pc, x == begin ? 2 * w : 2 * w + 1, lds);
        x = pc.next;
    }
}

// Joins the pieces of the units that a worker boundary cuts: workgroup x takes
// the unit that boundary x + 1 falls into, if it is the first one inside it;
// workgroups along y take kMergeRows rows each.
constexpr int kMergeRows = 32;

template <int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p) {
    extern __shared__ uint64_t s_tiles[];
    tile_prefix(p, s_tiles);
    const int64_t ptot = (int64_t)s_tiles[p.B] * p.Hkv;
    const int w = blockIdx.x + 1;
    const int64_t x = first_lane_int64(range_start(ptot, w, p.W, p.range_inv));
    const int64_t prev = first_lane_int64(range_start(ptot, w - 1, p.W, p.range_inv));
    if (x >= ptot || x == prev)
        return;
    const Piece pc = locate_tile(p, s_tiles, x, ptot);
    if (x == pc.us || prev > pc.us)
        return;   // not cut here, or an earlier boundary cuts it too
    const UnitSplit u = unit_split(ptot, pc.us, pc.n, p.W);
    const SeqInfo sq = seq_info(p, pc.b);
    constexpr int kPer = D / 8;   // values of a thread, eight threads per row
    const int r = blockIdx.y * kMergeRows + threadIdx.x / 8, part = threadIdx.x % 8;
    const int token = pc.m * p.TT + r / p.G;
    if (r >= p.TT * p.G || token >= sq.c.Q)
        return;
    float M = -INFINITY;
    for (int k = 0; k < u.nparts; k++)
        M = fmaxf(M, p.ws_lse[(int64_t)u.slot(k) * kTileRows + r]);
    float sum = 0.0f, o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; e++)
        o[e] = 0.0f;
    for (int k = 0; k < u.nparts; k++) {
        const int64_t row = (int64_t)u.slot(k) * kTileRows + r;
        const float lse = p.ws_lse[row];
        if (lse == -INFINITY)
            continue;
        const float a = fmaxf(fast_exp2(lse - M), kTiny);   // an infinite piece stays infinite
        sum += a;
#pragma unroll
        for (int e = 0; e < kPer; e += 4) {
            const f32x4_t x4 = *reinterpret_cast<const f32x4_t *>(p.ws_o + row * D + kPer * part + e);
#pragma unroll
            for (int i = 0; i < 4; i++)
                o[e + i] += a * x4[i];
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t *dst = p.out + (int64_t)(sq.row0 + token) * p.out_stride + (int64_t)(pc.g * p.G + r % p.G) * D + kPer * part;
#pragma unroll
    for (int e = 0; e < kPer; e += 4)
        *reinterpret_cast<uint2 *>(dst + e) =
            make_uint2(pack_bf16x2(o[e] * inv, o[e + 1] * inv), pack_bf16x2(o[e + 2] * inv, o[e + 3] * inv));
}

struct ChunkPlan {
    int G, TT, W;
    size_t ws_lse_off, ws_bytes;
};

int make_chunk_plan(const ts_chunk_shape *s, ChunkPlan *pl) {
    const int st = check_chunk_shape(s);
    if (st)
        return st;
    pl->G = s->num_q_heads / s->num_kv_heads;
    pl->TT = kTileRows / pl->G;
    // KV tiles of the call, from above
    const int64_t tiles = ((int64_t)s->num_tokens / pl->TT + std::min(s->num_seqs, s->num_tokens)) * s->num_kv_heads *
                          (((int64_t)s->max_ctx_len + kKeyTile - 1) / kKeyTile);
    pl->W = s->num_workers > 0 ? s->num_workers : (int)std::max<int64_t>(1, std::min<int64_t>(512, tiles / 2));
    const size_t rows = 2 * (size_t)pl->W * kTileRows;
    pl->ws_lse_off = rows * s->head_dim * sizeof(float);
    pl->ws_bytes = (pl->ws_lse_off + rows * sizeof(float) + 255) & ~(size_t)255;
    return TS_OK;
}

}  // namespace

int check_chunk_shape(const ts_chunk_shape *s) {
    if (!s)
        return fail(TS_ERR_NULL, "shape is NULL");
    if (s->num_seqs < 1 || s->num_seqs > kMaxSeqs)
        return fail(TS_ERR_SHAPE, "num_seqs %d outside [1, %d]", s->num_seqs, kMaxSeqs);
    if (s->num_tokens < 0 || s->num_tokens > (1 << 22))
        return fail(TS_ERR_SHAPE, "num_tokens %d outside [0, 2^22]", s->num_tokens);
    if (s->num_kv_heads < 1 || s->num_q_heads < 1 || s->num_q_heads % s->num_kv_heads)
        return fail(TS_ERR_SHAPE, "num_q_heads %d must be a positive multiple of num_kv_heads %d", s->num_q_heads,
                    s->num_kv_heads);
    if (s->num_q_heads / s->num_kv_heads > 16)
        return fail(TS_ERR_SHAPE, "group size %d exceeds 16", s->num_q_heads / s->num_kv_heads);
    if (s->num_q_heads > 1024)
        return fail(TS_ERR_SHAPE, "num_q_heads %d exceeds 1024", s->num_q_heads);
    if (s->head_dim != 64 && s->head_dim != 128)
        return fail(TS_ERR_SHAPE, "head_dim %d unsupported (64 or 128)", s->head_dim);
    if (s->page_size != kPage)
        return fail(TS_ERR_SHAPE, "page_size %d unsupported (16)", s->page_size);
    if (s->max_q_len < 0 || s->max_q_len > s->num_tokens)
        return fail(TS_ERR_SHAPE, "max_q_len %d outside [0, num_tokens]", s->max_q_len);
    if (s->max_pages_per_seq < 1 || s->max_pages_per_seq > (1 << 26))
        return fail(TS_ERR_SHAPE, "max_pages_per_seq %d outside [1, 2^26]", s->max_pages_per_seq);
    if (s->max_ctx_len < 1 || (int64_t)s->max_ctx_len > (int64_t)s->max_pages_per_seq * kPage)
        return fail(TS_ERR_SHAPE, "max_ctx_len %d outside [1, max_pages_per_seq x 16]", s->max_ctx_len);
    if (s->num_pages < 1 || s->num_pages > (1LL << 31))
        return fail(TS_ERR_SHAPE, "num_pages %lld outside [1, 2^31]", (long long)s->num_pages);
    if (s->num_workers < 0 || s->num_workers > (1 << 16))
        return fail(TS_ERR_SHAPE, "num_workers %d outside [0, 2^16]", s->num_workers);
    return TS_OK;
}

int check_stride(const char *name, int64_t stride, int64_t row) {
    if (stride < row || stride % 8 || stride > (1LL << 32))
        return fail(TS_ERR_ARG, "%s %lld must be a multiple of 8 of at least %lld elements", name, (long long)stride,
                    (long long)row);
    return TS_OK;
}

}  // namespace tsattn

using namespace tsattn;

extern "C" {

size_t ts_chunk_attn_workspace_size(const ts_chunk_shape *s) {
    clear_error();
    ChunkPlan pl;
    return make_chunk_plan(s, &pl) == TS_OK ? pl.ws_bytes : 0;
}

int ts_chunk_attn(const ts_chunk_shape *s, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                  const int32_t *page_table, const int32_t *ctx_lens, const int32_t *q_starts, void *out,
                  int64_t out_stride, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    ChunkPlan pl;
    int st = make_chunk_plan(s, &pl);
    if (st)
        return st;
    if (s->num_tokens == 0)
        return TS_OK;   // no rows, whose tensors may be NULL
    if (!q || !k_pages || !v_pages || !page_table || !ctx_lens || !q_starts || !out || !workspace)
        return fail(TS_ERR_NULL, "a pointer is NULL");
    if (!std::isfinite(scale))
        return fail(TS_ERR_ARG, "scale must be finite");
    if (workspace_bytes < pl.ws_bytes)
        return fail(TS_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, pl.ws_bytes);
    if ((((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)out) & 15) || ((uintptr_t)workspace & 255))
        return fail(TS_ERR_ARG, "misaligned pointer (tensors 16 B, workspace 256 B)");
    const int64_t row = (int64_t)s->num_q_heads * s->head_dim;
    if ((st = check_stride("q_stride", q_stride, row)) || (st = check_stride("out_stride", out_stride, row)))
        return st;
    if ((st = check_device()))
        return st;
    ChunkParams p;
    p.q = static_cast<const uint16_t *>(q);
    p.k_pages = static_cast<const uint16_t *>(k_pages);
    p.v_pages = static_cast<const uint16_t *>(v_pages);
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.q_starts = q_starts;
    p.out = static_cast<uint16_t *>(out);
    p.ws_o = static_cast<float *>(workspace);
    p.ws_lse = reinterpret_cast<float *>(static_cast<char *>(workspace) + pl.ws_lse_off);
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.num_pages = s->num_pages;
    p.B = s->num_seqs;
    p.Hq = s->num_q_heads;
    p.Hkv = s->num_kv_heads;
    p.G = pl.G;
    p.max_pages = s->max_pages_per_seq;
    p.num_tokens = s->num_tokens;
    p.TT = pl.TT;
    p.W = pl.W;
    p.range_inv = range_reciprocal(pl.W);
    p.scale_log2 = std::fabs(scale) * 1.44269504088896341f;
    p.q_sign = std::signbit(scale) ? 0x80008000u : 0u;
    const size_t pre = (((size_t)s->num_seqs + 1) * 8 + 127) & ~(size_t)127;
    const bool small = s->head_dim == 64;
    const auto main_k = small ? chunk_attn_kernel<64> : chunk_attn_kernel<128>;
    const auto merge_k = small ? chunk_merge_kernel<64> : chunk_merge_kernel<128>;
    hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(main_k, dim3((unsigned)pl.W), dim3(kChunkWaves * kWave),
                       pre + (small ? Chunk<64>::kLds : Chunk<128>::kLds), hs, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return hip_fail(e, "chunk attention launch");
    if (pl.W > 1) {
        hipLaunchKernelGGL(merge_k, dim3((unsigned)pl.W - 1, kTileRows / kMergeRows), dim3(256), pre, hs, p);
        if ((e = hipGetLastError()) != hipSuccess)
            return hip_fail(e, "chunk merge launch");
    }
    return TS_OK;
}

}  // extern "C"
