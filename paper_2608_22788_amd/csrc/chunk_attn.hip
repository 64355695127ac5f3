// chunk_attn.hip -- attention of chunks of new tokens over the paged cache: any
// number of packed rows per sequence, from one decoding token to a whole prompt.
//
// For row i of a sequence (Q new tokens, context length L) and query head h:
//   out = sum_t w_t V_t / sum_t w_t,  w_t = exp(scale <q, K_t>),  t <= L - Q + i.
// In one pass over the keys, in units of log2: with a reference m that is at
// least the largest score so far less 8, w_t = 2^(s_t - m); where a score passes
// m + 8, m moves up to it and what is summed so far is scaled by 2^(old - new).
// Weights stay at 2^8 or below; they are rounded to bf16 for the second matrix
// product, which takes no more, and their float32 sum takes the rounded ones too,
// so that the result stays an average of values (two to an instruction).  That
// rounding is a choice: outputs are off by 2.1-2.3e-3 (rel-L2 against 64 bits),
// of which the rounding of the result alone is 1.6-1.7e-3; a second product with
// what it takes away brings that back and takes a prompt from 524 to 708 us, four
// resumed rollouts from 436 to 575, a mixed batch from 77 to 86.
//
// Work.  A row tile is 256 rows of one KV head (256 / G tokens with their G query
// heads each, so that a key is read once for the group), a KV tile 64 keys.  A
// workgroup of 8 wavefronts, one per CU, holds 32 rows per wavefront: q, the
// running sums and the output in registers.  The KV tiles of all row tiles form
// one line that is cut into W equal ranges (chunk_partition.h), so a ragged batch
// and a causal prompt load all CUs alike whatever their lengths; a row tile that
// a boundary cuts leaves its pieces, normalised, with their log2-sum-exp in the
// workspace, and chunk_merge_kernel joins them.
//
// Scores are computed transposed, S^T = K Q^T (32 x 32 x 16 products), so that
// a lane holds scores of one row and its weights are already where the second
// product O^T += V^T P^T takes them from; V^T is read by the transposing LDS
// read.  Tiles come to LDS by loads that pass no registers, four stages deep, and
// rows are stored in an order without bank conflicts (measured: none).
//
// What bounds it.  Long chunks: 4 D operations per row and key.  At 8,192 tokens
// of a prompt, 32/8 heads, head_dim 128: 521-557 us by box, 990-1,055 TFLOP/s,
// 72-77 % of what a 16384^3 bf16 product reaches on the card.  The clock is about
// 2 GHz; of a SIMD's cycles the matrix unit is busy 53 %, and other vector
// instructions (an exponential, which takes two issue slots, a multiply-add and
// half a maximum, a packing and a sum for each score) issue in 39 % (how far the
// two overlap the counters do not say).  What mattered, on that case:
//   - 128 rows on 4 wavefronts took 781 us: every CU then draws 10 TB/s of tiles
//     through the L2s, which alone take 423 us; 256 rows halve that;
//   - a tile's weights beside the next tile's scores, in a fixed order: 551 us
//     (577 in the order that the compiler chose);
//   - weights summed two at a time: 428 -> 423 us with four resumed rollouts;
//   - no effect: more of the weights beside the scores, wave priorities, operands
//     read six products ahead instead of four; worse: two wavefronts to the halves
//     of one tile (564 instead of 555), 64 rows per wavefront (726 instead of 522).
// head_dim 64 has twice the exponentials per operation: 92-95 us for 56.9 GFLOP;
// matrix unit 31 %, other vector instructions 47 % of a busy CU's cycles, and CUs
// have work for 82 % of the kernel's time only (starts, ends).
// Long caches under few rows: the cache's bytes, 16 KiB of K and as much of V per
// tile.  32 sequences, most of them decoding behind up to 4,000 tokens: 77 us for
// 317 MB; 256 sequences of one token behind 1,000: 181 us for 1,057 MB, 5.8 TB/s.
// One short chunk (37 tokens behind 2,011, 23 us): the chain of a launch, finding
// the work, two tiles and the join of 16 pieces.
//
// The cache held in 8 bits (kv8_common.h).  The same kernel; only the tiles' way
// differs: codes come to LDS as they are, four tiles deep, each wavefront turns the
// page that it loaded into bf16 rows of a stage, in registers, two codes to an
// instruction that takes the page's power along (exact), and two stages suffice.
// Half of the bytes, and for each value half a conversion and an eighth of an LDS
// store, 6 % of the time in bank conflicts.  A prompt of 8,192 tokens takes 546-565 us,
// 973-1,007 TFLOP/s (538-563 from the bf16 cache on the same boxes; on another 553
// against 521), 16 ragged prompts of up to 1,024 tokens 308-315 us.  What mattered, on
// the prompt: conversions by all wavefronts at the start of a step 585 us; the keys'
// wavefronts before and the values' after it 558; ids and powers of 64 tiles in a lane
// each 548.
// Row tiles of up to 16 rows (decoding sequences) would have one busy wavefront of
// eight and take 1.2 us a KV tile, as long as from the bf16 cache, whose bytes take
// that long.  Their wavefronts share the keys instead (few_rows): 0.66 us, 6.3 TB/s
// over the chip.  32 mixed sequences, 138 MB: 83 us without, 77 with the places of the
// bf16 cache, 63 with those that the times of either kind ask for (chunk_partition.h).
// The kernel of head_dim 128 keeps 8 registers in scratch for it (36 bytes a lane; two
// reloads are in the loop over these row tiles' keys), and a prompt takes 1 % longer
// (554 -> 561 on one box); with three steps under way for a wavefront instead of two
// it would be 20 registers, and 79 us.  A piece starts cold, so
// contexts of a few tiles gain nothing from their half of the bytes: 160 sequences
// of one token behind 64 take 32 us (26-27 from the bf16 cache), behind 128 both 35,
// behind 256 43 against 50, behind 4,096 247 against 406.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_common.h"
#include "attn_verify.h"
#include "chunk_common.h"
#include "chunk_partition.h"
#include "kv8_common.h"
#include "ts_attn.h"
#include "ts_internal.h"

namespace tsattn {

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kRowBlock = 32;      // rows of a matrix-core tile
constexpr int kChunkWaves = 8;
// KV tiles in LDS: one in use, the others on their way.  Of the cache held in 8
// bits: as bf16, the values in use with the keys of the next tile, and the place of
// those after them; and as codes, on their way.  Both take 128 KiB at head_dim 128.
constexpr int stages(bool k8) { return k8 ? 2 : 4; }
constexpr int kCodeStages = 4;
static_assert(kTileRows == kChunkWaves * kRowBlock, "a row block per wavefront");
constexpr float kTiny = 1.17549435e-38f;   // the smallest normal float32
constexpr float kLowest = -3.0e38f;       // the reference of a row without a score yet
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
    struct Cut *cuts;           // [W] the unit at the start of each worker's range
    int64_t q_stride, out_stride, num_pages;
    int B, Hq, Hkv, G, max_pages, num_tokens;
    int TT;                     // tokens per row tile
    int W;                      // workers
    uint32_t range_inv;
    float scale_log2;           // |scale| * log2(e)
    uint32_t q_sign;            // sign bits to flip in a pair of q values
    const uint8_t *kv_scales;   // [num_pages][Hkv][2] (the cache held in 8 bits, whose pages hold bytes)
};

// Sequence b: its first packed row, new tokens and tokens in front of them.
// Row and length limits keep every access in bounds whatever the arrays hold.
struct SeqInfo {
    int row0, L;
    ChunkSeq c;
};
template <bool k8>
__device__ __forceinline__ SeqInfo seq_info(const ChunkParams &p, int b) {
    SeqInfo s;
    const int a = min(max(ld_meta(p.q_starts, b), 0), p.num_tokens);
    const int e = min(max(ld_meta(p.q_starts, b + 1), 0), p.num_tokens);
    s.row0 = a;
    s.c.Q = max(e - a, 0);
    s.L = clamped_len(ld_meta(p.ctx_lens, b), p.max_pages);
    s.c.P = max(s.L - s.c.Q, 0);
    s.c.TT = p.TT;
    s.c.G = p.G;
    s.c.k8 = k8;
    return s;
}

// Places of one head up to the end of each sequence, in s_end[0 .. B - 1]: a
// thread per sequence, sums within wavefronts and then, past 64 sequences, over
// them.  (With one wavefront for all of them a call of 4,096 sequences of 100
// tokens took 113 us more; it takes 720.)
template <bool k8>
__device__ inline void tile_ends(const ChunkParams &p, uint64_t *s_end) {
    const int wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    uint64_t base = 0;
    for (int b0 = 0; b0 < p.B; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        uint64_t n = 0;
        if (b < p.B) {
            const SeqInfo s = seq_info<k8>(p, b);
            n = s.c.Q > 0 ? (uint64_t)s.c.total() : 0;
        }
        const uint64_t incl = wave_incl_scan(n);
        if (b < p.B)
            s_end[b] = incl;
        if (p.B <= kWave)
            break;
        __syncthreads();
        uint64_t before = base;
        for (int i = 0; i < waves && b0 + i * kWave < p.B; i++) {
            const uint64_t sum = s_end[min(b0 + i * kWave + kWave - 1, p.B - 1)];
            before += i < wave ? sum : 0;
            base += sum;
        }
        __syncthreads();
        if (b < p.B)
            s_end[b] = before + incl;
    }
    __syncthreads();
}

// What joins the pieces of the unit that holds the first place of a worker's
// range, as chunk_merge_kernel needs it (which took 16.7 us for 32 mixed
// sequences when it searched the unit itself, so 8.6).
struct Cut {
    int64_t ptot, us;  // places of the call, and in front of the unit
    int n, weight;     // KV tiles of the unit, and places of each
    int row, tokens;   // its first packed row, and its tokens
    int head;          // and first query head
};

struct Piece {
    int b, g, m;       // sequence, KV head, row tile
    int j0, j1;        // KV tiles [j0, j1) of it
    int n, weight;     // KV tiles of the whole unit, and places of each
    bool whole;
    int64_t us;        // global index of the unit's first place
    int64_t next;      // and of the first one behind the piece
};

// The tiles of unit r.us, r.m (of sequence c) in places [from, range_end).
__device__ __forceinline__ void cut_piece(Piece &r, const ChunkSeq &c, int64_t from, int64_t range_end) {
    r.n = first_lane_int(c.cost(r.m));
    r.weight = first_lane_int(c.weight(r.m));
    const int64_t unit_end = r.us + (int64_t)r.n * r.weight + c.behind(r.m);
    r.next = unit_end < range_end ? unit_end : range_end;
    r.j0 = first_lane_int(min(tile_at(from - r.us, r.weight), r.n));
    r.j1 = first_lane_int(min(tile_at(r.next - r.us, r.weight), r.n));
    r.whole = r.j0 == 0 && r.j1 == r.n;
}

// The unit that holds place x, and the part of it in [x, range_end).
// Units are laid out sequence by sequence, head by head, row tile by row tile.
template <bool k8>
__device__ inline Piece locate_tile(const ChunkParams &p, const uint64_t *s_end, int64_t x, int64_t range_end) {
    const int lane = threadIdx.x & (kWave - 1);
    Piece r;
    // the first sequence that ends behind x
    int lo = 0, n = p.B;
    const auto before = [&](int b) { return (int64_t)s_end[min(b, p.B - 1)] * p.Hkv <= x; };
    if (p.B > kWave) {
        const int step = (p.B + kWave - 1) / kWave, last = (lane + 1) * step - 1;
        lo = step * __popcll(__ballot(last < p.B && before(last)));
        n = min(step, p.B - lo);
    }
    r.b = first_lane_int(min(lo + __popcll(__ballot(lane < n && before(lo + lane))), p.B - 1));
    const int64_t pre = r.b ? first_lane_int64((int64_t)s_end[r.b - 1]) : 0;
    const int64_t per_head = first_lane_int64((int64_t)s_end[r.b]) - pre;
    const int64_t off = x - pre * p.Hkv;
    r.g = first_lane_int((int)(off / per_head));
    const int64_t in_head = off - r.g * per_head;
    const ChunkSeq c = seq_info<k8>(p, r.b).c;
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
    r.us = x - in_head + start;
    cut_piece(r, c, x, range_end);
    return r;
}

// The next piece with KV tiles at or behind x in a worker's range, false if
// there is none.  `r` is the piece before it, whether it has tiles or not: the
// row tiles of one head follow each other, so most of the time nothing is searched.
template <bool k8>
__device__ __forceinline__ bool next_piece(const ChunkParams &p, const uint64_t *s_end, int64_t &x, int64_t range_end, Piece &r) {
    while (x < range_end) {
        const ChunkSeq c = seq_info<k8>(p, r.b).c;
        if (r.m + 1 < c.tiles() || r.g + 1 < p.Hkv) {
            const bool same = r.m + 1 < c.tiles();
            r.g = same ? r.g : r.g + 1;
            r.m = same ? r.m + 1 : 0;
            r.us = x;
            cut_piece(r, c, x, range_end);
        } else {
            r = locate_tile<k8>(p, s_end, x, range_end);
        }
        x = r.next;
        if (r.j0 < r.j1)
            return true;
    }
    return false;
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

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;

// Loads kLoads blocks of 1 KiB into LDS without passing registers: block i from
// byte (from ^ (twist i)) + 1024 i of the resource (each lane 16 bytes), to `to`
// + 1024 i + 16 lane.  The instructions have no outputs, so nothing can be taken
// for written before it is; m0, which they need, is named as overwritten.
// Completion is counted by vmcnt: dma_wait() and a barrier come before the data
// is read.
//
// Keys that one row tile alone reads (kOnce) are loaded as not to be kept: 256
// sequences of one token behind 1,000 take 181 us so, 198 otherwise; a prompt,
// whose row tiles find each other's keys in the L2, would take 588 instead of 519.
template <int kLoads, bool kOnce>
__device__ __forceinline__ void dma_blocks(block_rsrc_t rsrc, uint32_t to, int from, int twist) {
    static_assert(kLoads == 1 || kLoads == 2 || kLoads == 4, "blocks");
#define TS_DMA_BLOCK(reg, offset, kept) "buffer_load_dwordx4 %" reg ", %1, 0 offen offset:" offset kept " lds\n\t"
#define TS_DMA_BLOCKS(kept)                                                                                            \
    if constexpr (kLoads == 4)                                                                                         \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t" TS_DMA_BLOCK("2", "0", kept) TS_DMA_BLOCK("3", "1024", kept)    \
                         TS_DMA_BLOCK("4", "2048", kept) TS_DMA_BLOCK("5", "%6", kept)::"s"(to), "s"(rsrc), "v"(from), \
                     "v"(from ^ twist), "v"(from ^ 2 * twist), "v"(from ^ 3 * twist), "n"(3 * 1024)                    \
                     : "m0", "memory");                                                                                \
    else if constexpr (kLoads == 2)                                                                                    \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t" TS_DMA_BLOCK("2", "0", kept)                                   \
                         TS_DMA_BLOCK("3", "1024", kept)::"s"(to), "s"(rsrc), "v"(from), "v"(from ^ twist)             \
                     : "m0", "memory");                                                                                \
    else                                                                                                               \
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t" TS_DMA_BLOCK("2", "0", kept)::"s"(to), "s"(rsrc), "v"(from)    \
                     : "m0", "memory")
    // (a clobber of m0 warns that its value is not kept: nobody needs it)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    if constexpr (kOnce) {
        TS_DMA_BLOCKS(" nt");
    } else {
        TS_DMA_BLOCKS("");
    }
#pragma clang diagnostic pop
#undef TS_DMA_BLOCKS
#undef TS_DMA_BLOCK
}
// Waits until at most the loads of the last `later` tiles are under way.
template <int kLoads>
__device__ __forceinline__ void dma_wait(int later) {
    static_assert(stages(false) == 4 && kCodeStages == 4, "up to three later tiles");
    if (later >= 3)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * kLoads) : "memory");
    else if (later == 2)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
    else if (later == 1)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int D, bool k8>
struct Chunk {
    static constexpr int kStages = stages(k8);
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kPieces = kRowBytes / 16;         // 16-byte pieces of a row
    static constexpr int kKBytes = kKeyTile * kRowBytes;   // the keys of a stage; the values follow
    static constexpr int kStage = 2 * kKBytes;
    static constexpr int kCodeBytes = k8 ? 2 * kKeyTile * D : 0;   // keys and values of a tile as codes
    static constexpr int kCodes = kStages * kStage;        // where they begin
    static constexpr int kLds = kCodes + kCodeStages * kCodeBytes;
    static constexpr int kPageBytes = k8 ? kPage * D : kPage * kRowBytes;   // of one (page, KV head) block in memory
    static constexpr int kLoads = kPageBytes / (16 * kWave);   // loads of a wave per page block
    static constexpr int kKSteps = D / 16;
    static constexpr int kDTiles = D / 32;

    // Row `key` of a tile is stored with its 16-byte pieces in an order that
    // depends on the key, so that reads of one column of many rows spread over
    // the 64 banks.  Keys: 32 lanes read a piece of a row each, 16 bytes, and
    // the sixteen that are served together have sixteen different keys modulo
    // 16.  Values: 32 lanes read 32 bytes of four consecutive rows, at two
    // places.  (Rows of 128 bytes: two fill the banks once.)
    __device__ __forceinline__ static int k_piece(int key, int piece) { return piece ^ (D == 128 ? key & 15 : key >> 1 & 7); }
    __device__ __forceinline__ static int v_piece(int key, int piece) { return piece ^ (D == 128 ? 4 * (key & 3) : 4 * (key >> 1 & 1)); }

    struct State {
        u32x4_t qf[kKSteps];
        f32x16_t o[kDTiles];
        float m_ref, l;
        int lim;                  // keys that this lane's row sees
        // this lane's LDS addresses in stage 0, of the first keys and values
        uint32_t k, v;
        int from, twist;          // and where in a page it loads from (dma_blocks)
        uint32_t to;              // where it stores the first of its codes as bf16, in stage 0
    };

    // Starts loading a wavefront's part of a tile, the keys (wavefronts 0 to 3)
    // or values of a page, to `stage`.  A page outside the pool is stored as zeros;
    // what is under way then arrives first, so that counts of loads stay counts of
    // tiles.
    __device__ __forceinline__ static void dma_page(const ChunkParams &p, const State &st, int pid, bool once, int g, char *stage, int wave, int lane) {
        char *to = stage + wave * kPageBytes;   // (the values follow the keys)
        if (__builtin_expect(pid < 0 || pid >= p.num_pages, 0)) {
            dma_wait<kLoads>(0);
#pragma unroll
            for (int i = 0; i < kLoads; i++)
                *reinterpret_cast<u32x4_t *>(to + 16 * (i * kWave + lane)) = u32x4_t{0u, 0u, 0u, 0u};
            return;
        }
        const size_t block = (size_t)pid * p.Hkv + g;
        const char *pages = reinterpret_cast<const char *>(wave < kTilePages ? p.k_pages : p.v_pages);
        const block_rsrc_t rsrc = block_rsrc(pages + block * kPageBytes, kPageBytes);
        const uint32_t at = (uint32_t)first_lane_int((int)(uintptr_t)(lds_char *)to);
        if (once)
            dma_blocks<kLoads, true>(rsrc, at, st.from, st.twist);
        else
            dma_blocks<kLoads, false>(rsrc, at, st.from, st.twist);
    }

    // A wavefront's page of a tile from codes to bf16, times its power (exact), in the
    // order in which rows are stored: a lane takes back the 16 codes that it loaded,
    // two pieces of a row.  With `clean`, NaN codes are replaced by zero; returns
    // whether one of the first `rows` rows held one (the others are not in the
    // context).
    __device__ __forceinline__ static bool convert_page(const State &st, const char *codes, int stage, float power, bool clean, int rows, int wave,
                                                        int lane) {
        constexpr int kLanes = D / 16;   // lanes of a row
        bool any = false;
        u32x4_t c[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            c[i] = *reinterpret_cast<const u32x4_t *>(codes + 16 * lane + 1024 * i);
        if (__builtin_expect(clean, 0)) {
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                uint32_t odd = 0;
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    const uint32_t m = ((c[i][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                    c[i][w] &= ~((m >> 7) * 0xffu);
                    odd |= m;
                }
                any |= odd && i * (kWave / kLanes) + lane / kLanes < rows;
            }
        }
        // Block i holds rows 8 i .. of head_dim 128, whose key pieces differ by 8 i.
        const uint32_t twist = wave < kTilePages ? 128 : 0;
#pragma unroll
        for (int i = 0; i < kLoads; i++)
#pragma unroll
            for (int u = 0; u < 2; u++) {
                u32x4_t x;
#pragma unroll
                for (int w = 0; w < 4; w++)
                    x[w] = __builtin_bit_cast(uint32_t, w % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i][2 * u + w / 2], power, true)
                                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i][2 * u + w / 2], power, false));
                lds_char *at = (lds_char *)(uintptr_t)((st.to ^ (16 * u + twist * i)) + stage * kStage);
                *(lds_u32x4 *)(at + i * (kWave / kLanes) * kRowBytes) = x;
            }
        return any;
    }

    __device__ __forceinline__ static void set_addresses(State &st, char *lds, int wave, int lane) {
        const int n = lane & 31, h = lane >> 5;
        const uint32_t base = (uint32_t)(uintptr_t)(lds_char *)lds;
        st.k = base + n * kRowBytes + 16 * k_piece(n, h);
        // Value operand.  ds_read_b64_tr_b16 hands lane i of 16 lanes element
        // i % 4 of the 8 bytes that lane 4 k + i / 4 addresses, as element k;
        // so with lane i addressing key i / 4, dimensions 4 (i % 4) .. + 3 of
        // 16, it receives four keys of dimension i.
        const int i = lane & 15, x = i >> 2;
        st.v = base + kKBytes + (4 * h + x) * kRowBytes + 16 * v_piece(x, 2 * ((lane >> 4) & 1)) + 8 * (i & 3);
        // Block i of 1 KiB of a page holds its rows (64 / kPieces) i + lane /
        // kPieces in stored order: the exchange of key pieces differs by 4 i,
        // 64 i bytes, that of value pieces not at all.
        // (Codes are loaded in the order of the page.)
        const int row = lane / kPieces, piece = lane % kPieces;
        const bool keys = wave < kTilePages;
        st.from = k8 ? 16 * lane : row * kRowBytes + 16 * (keys ? k_piece(row, piece) : v_piece(row, piece));
        st.twist = keys && !k8 ? 64 : 0;
        const int code_row = lane / (D / 16), code_piece = 2 * (lane % (D / 16));
        st.to = base + (wave * kPage + code_row) * kRowBytes +
                16 * (keys ? k_piece(code_row, code_piece) : v_piece(code_row, code_piece));
    }

    // Keys 32 kt .. + 31, dimensions 16 ks .. + 15.
    __device__ __forceinline__ static bf16x8_t k_frag(const State &st, int stage, int kt, int ks) {
        const lds_char *at = (const lds_char *)(uintptr_t)((st.k + stage) ^ (32 * ks));
        return __builtin_bit_cast(bf16x8_t, *(const lds_u32x4 *)(at + 32 * kRowBytes * kt));
    }
    // Dimensions 32 dt .. + 31 of the 16 keys of a step, in the order in which
    // a lane's score registers hold them: 4 h .. + 3 and 8 + 4 h .. + 3.
    __device__ __forceinline__ static bf16x8_t v_frag(const State &st, int stage, int dt, int step) {
        const lds_char *at = (const lds_char *)(uintptr_t)((st.v + stage) ^ (64 * dt)) + 16 * kRowBytes * step;
        s16x4_t ab[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at),
                         __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * kRowBytes))};
        return __builtin_bit_cast(bf16x8_t, ab);
    }

    struct Scores {
        f32x16_t s[2];   // keys 32 kt + 8 (e / 4) + 4 h + e % 4 of this lane's row in s[kt][e]
        float mx;        // the largest, times the scale
    };

    // Raises the reference where a score exceeds it by more than the slack.
    __device__ __forceinline__ static void raise(State &st, float mx) {
        if (__builtin_expect(__any(mx > st.m_ref + kRescaleSlack), 0)) {
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
    }

    __device__ __forceinline__ static void scores(const State &st, int stage, Scores &n) {
#pragma unroll
        for (int kt = 0; kt < 2; kt++) {
            f32x16_t s = {};
#pragma unroll
            for (int ks = 0; ks < kKSteps; ks++)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(st, stage, kt, ks), __builtin_bit_cast(bf16x8_t, st.qf[ks]), s, 0, 0, 0);
            n.s[kt] = s;
        }
    }
    // Scores of keys that the row does not see: their weight is exactly zero,
    // since the reference is finite.
    __device__ __forceinline__ static void mask(Scores &n, int room) {
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int e = 0; e < 16; e++)
                n.s[kt][e] = 32 * kt + 8 * (e / 4) + e % 4 < room ? n.s[kt][e] : -INFINITY;
    }
    __device__ __forceinline__ static void largest(const ChunkParams &p, Scores &n) {
        float m = fmaxf(n.s[0][0], n.s[0][1]);
#pragma unroll
        for (int e = 2; e < 32; e += 2)
            m = fmaxf(fmaxf(m, n.s[e / 16][e % 16]), n.s[e / 16][e % 16 + 1]);
        n.mx = m * p.scale_log2;
    }

    // One KV tile, whose scores are `c`, and (kNext) the scores `n` of the next
    // one.  `room` (masked): keys of the tile that the lane's row sees, less 4 h.
    template <bool kNext>
    __device__ __forceinline__ static void tile_step(const ChunkParams &p, State &st, Scores &c, Scores &n, int v_stage, int k_stage,
                                     bool masked, int room) {
        if (__builtin_expect(masked, 0)) {
            mask(c, room);
            largest(p, c);
        }
        raise(st, c.mx);
        // From here on nothing branches, and the order of the instructions is
        // the one written here (sched_fence): each matrix product is followed by
        // the vector instructions that fit beside it and the operand of the
        // product four later.  The next scores' products stand beside the
        // weights of the first 32 keys, the value products beside those of the
        // other 32, then the next maximum.
        constexpr int kAhead = 4, kScore = 2 * kKSteps, kValue = 4 * kDTiles;
        u32x4_t pf[2][2];
        bf16x8_t kf[kAhead], vf[kAhead];
        float x[2][16], sum[2] = {0.0f, 0.0f}, m[2] = {-INFINITY, -INFINITY};
        const auto weigh = [&](int half, int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int e = from; e < to; e++) {
                x[half][e] = fast_exp2(__builtin_fmaf(c.s[half][e], p.scale_log2, -st.m_ref));
                if (e % 2) {
                    pf[half][e / 8][e / 2 % 4] = pack_bf16x2(x[half][e - 1], x[half][e]);
                    sum[e / 2 % 2] = dot2_bf16(pf[half][e / 8][e / 2 % 4], 0x3f803f80u, sum[e / 2 % 2]);
                }
            }
            asm volatile("" : "+v"(sum[0]), "+v"(sum[1]));   // (here, not at the end of the step: 1.7 %)
        };
        const auto values = [&](int i) { return v_frag(st, v_stage, i % kDTiles, i / kDTiles); };
        if constexpr (kNext) {
            const f32x16_t zero = {};
            n.s[0] = n.s[1] = zero;
#pragma unroll
            for (int i = 0; i < kAhead; i++)
                kf[i] = k_frag(st, k_stage, i / kKSteps, i % kKSteps);
            sched_fence();
#pragma unroll
            for (int i = 0; i < kScore; i++) {
                n.s[i / kKSteps] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % kAhead], __builtin_bit_cast(bf16x8_t, st.qf[i % kKSteps]),
                                                                           n.s[i / kKSteps], 0, 0, 0);
                if (i + kAhead < kScore)
                    kf[i % kAhead] = k_frag(st, k_stage, (i + kAhead) / kKSteps, (i + kAhead) % kKSteps);
                else
                    vf[i + kAhead - kScore] = values(i + kAhead - kScore);
                weigh(0, i * 16 / kScore, (i + 1) * 16 / kScore);
                sched_fence();
            }
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; i++)
                vf[i] = values(i);
            weigh(0, 0, 16);
        }
#pragma unroll
        for (int i = 0; i < kValue; i++) {
            f32x16_t &o = st.o[i % kDTiles];
            const int step = i / kDTiles;
            o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % kAhead], __builtin_bit_cast(bf16x8_t, pf[step / 2][step % 2]), o, 0, 0, 0);
            if (i + kAhead < kValue)
                vf[i % kAhead] = values(i + kAhead);
            if (i < kValue / 2)
                weigh(1, i * 32 / kValue, (i + 1) * 32 / kValue);
            else if constexpr (kNext) {
#pragma unroll
                for (int e = (i - kValue / 2) * 64 / kValue; e < (i - kValue / 2 + 1) * 64 / kValue; e += 2)
                    m[e / 2 % 2] = fmaxf(fmaxf(m[e / 2 % 2], n.s[e / 16][e % 16]), n.s[e / 16][e % 16 + 1]);
                asm volatile("" : "+v"(m[0]), "+v"(m[1]));
            }
            sched_fence();
        }
        st.l += sum[0] + sum[1];
        if constexpr (kNext)
            n.mx = fmaxf(m[0], m[1]) * p.scale_log2;
    }

    // Infinite and NaN values.  Where a row does not see a key, the key's zero
    // weight would still make NaN of such a value in the matrix product.  So in
    // the tiles that some row of the unit does not see whole (the last one to
    // three) they are replaced by zero in LDS before the tile is used, and put
    // back afterwards for the rows that see them, whose result is infinite or NaN
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

    // The values of the page that this wavefront has loaded; returns whether one
    // of its first `rows` rows held such a value (the others are not in the context).
    __device__ __forceinline__ static bool clean_page(char *stage, int wave, int lane, int rows) {
        char *page = stage + wave * (kPage * kRowBytes);
        bool any = false;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            u32x4_t *at = reinterpret_cast<u32x4_t *>(page + 16 * (i * kWave + lane));
            u32x4_t v = *at;
            const bool odd = clear_odd(v);
            if (odd)
                *at = v;
            any |= odd && (i * kWave + lane) / kPieces < rows;
        }
        return any;
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
            const size_t at = (((size_t)pid * p.Hkv + g) * kPage + t % kPage) * D + 4 * h;
            if (t >= st.lim)
                continue;
            if constexpr (k8) {
                const uint8_t *row = reinterpret_cast<const uint8_t *>(p.v_pages) + at;
#pragma unroll
                for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const uint32_t x = *reinterpret_cast<const uint32_t *>(row + 32 * dt + 8 * e);
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if ((x >> 8 * i & 0x7f) == 0x7f)
                                st.o[dt][4 * e + i] = __uint_as_float(0x7fc00000u);
                    }
                continue;
            }
            const uint16_t *row = p.v_pages + at;
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

    // The ids of a wavefront's pages in consecutive tiles, read four at a time as
    // scalars (a vector load would have to wait for every page under way).
    struct Pages {
        const int32_t *pt;
        int first, last;   // page of the first tile; the last page of the context
        bool once;         // no other row tile reads them
        int ids[4];
        __device__ __forceinline__ int next(int i) {   // tiles i = 0, 1, ... of the piece, in order
            if (i % 4 == 0)
#pragma unroll
                for (int k = 0; k < 4; k++)
                    ids[k] = ld_meta(pt, min(first + (i + k) * kTilePages, last));
            const int lo = i & 1 ? ids[1] : ids[0], hi = i & 1 ? ids[3] : ids[2];
            return first_lane_int(i & 2 ? hi : lo);
        }
    };
    // Of codes, a lane holds one of 64 tiles: the id of the wavefront's page and the
    // byte of its power, which reach their tile by lane reads.  (Scalar loads of them
    // tile by tile would make every wait for LDS a wait for memory, since both are
    // counted together: 16 ragged sequences 321 us instead of 313.)
    struct CodePages {
        const int32_t *pt;
        int first, last;   // as above
        bool once;
        int ids;           // of the 64 tiles of the next tile to be loaded
        int bytes, later;  // of those of the next one to be converted, and of `ids`
        __device__ __forceinline__ void fetch(const ChunkParams &p, int i, int g, int wave, int lane) {   // tiles i .. i + 63
            const int pid = pt[min(first + (i + lane) * kTilePages, last)];
            ids = pid;
            later = 127;
            if (pid >= 0 && pid < p.num_pages)
                later = p.kv_scales[((size_t)pid * p.Hkv + g) * 2 + (wave < kTilePages ? 0 : 1)];
        }
        __device__ __forceinline__ int id(int i) const { return __builtin_amdgcn_readlane(ids, i % kWave); }
        __device__ __forceinline__ float power(int i) const { return power_of(__builtin_amdgcn_readlane(bytes, i % kWave)); }
    };

    // Starts loading the first tiles of a piece.
    typedef std::conditional_t<k8, CodePages, Pages> TilePages;
    __device__ __forceinline__ static TilePages start(const ChunkParams &p, const State &st, const Piece &pc, char *lds, int wave, int lane) {
        const SeqInfo sq = seq_info<k8>(p, pc.b);
        TilePages pages{p.page_table + (size_t)pc.b * p.max_pages, first_lane_int(pc.j0 * kTilePages + wave % kTilePages),
                    first_lane_int((max(sq.L, 1) - 1) / kPage), sq.c.Q <= sq.c.TT};
        if constexpr (k8) {
            pages.fetch(p, 0, pc.g, wave, lane);
            pages.bytes = pages.later;
#pragma unroll
            for (int i = 0; i < kCodeStages; i++)
                if (i < pc.j1 - pc.j0)
                    dma_page(p, st, pages.id(i), pages.once, pc.g, lds + kCodes + i * kCodeBytes, wave, lane);
        } else {
            const int n = min(pc.j1 - pc.j0, kStages - 1);
            for (int i = 0; i < n; i++)
                dma_page(p, st, pages.next(i), pages.once, pc.g, lds + i * kStage, wave, lane);
        }
        return pages;
    }

    // ---- row tiles of up to 16 rows, of the cache held in 8 bits ------------------
    // One wavefront has rows then, so the wavefronts take turns at the keys instead:
    // wavefront w the pages 2 w, 2 w + 1 of every 16, in the steps of attn_verify.h,
    // straight to registers, one step ahead.  Their sums meet in LDS.
    typedef Verify<D, 1, true> Few;
    __device__ __forceinline__ static bool is_few(const ChunkParams &p, const Piece &pc) {
        const SeqInfo sq = seq_info<k8>(p, pc.b);
        return k8 && first_lane_int(min(p.TT, sq.c.Q - pc.m * p.TT) * p.G) <= kFewRows;
    }
    __device__ __forceinline__ static void few_rows(const ChunkParams &p, const Piece &pc, int slot, char *lds, int wave, int lane) {
        constexpr int kFewPages = 2, kSteps = kWave / kFewPages, kRing = 2, VE = D / 16;
        static_assert(Few::kStep == kFewPages, "pages of a step");
        // (Unknown here, so that no address of this function is worked out in front of
        // the loop over pieces and held through the other row tiles' steps.)
        asm volatile("" : "+v"(lane));
        const SeqInfo sq = seq_info<k8>(p, pc.b);
        const int n = lane & 15, kq = lane >> 4;
        const int rows = first_lane_int(min(p.TT, sq.c.Q - pc.m * p.TT) * p.G);
        const int seg_end = first_lane_int(min(sq.L, pc.j1 * kKeyTile));
        const int first_lim = first_lane_int(sq.L - sq.c.Q + pc.m * p.TT + 1);
        const int first = pc.j0 * kTilePages, end = first_lane_int((max(seg_end, 0) + kPage - 1) / kPage);
        const int steps = max(end - first + kFewPages - 1, 0) / kFewPages;
        const int own = steps > wave ? (steps - wave + kChunkWaves - 1) / kChunkWaves : 0;
        const auto page_of = [&](int s) { return first + kFewPages * (wave + kChunkWaves * s); };

        // Page ids and powers of 32 steps, one page in a lane each.
        const int32_t *pt = p.page_table + (size_t)pc.b * p.max_pages;
        int ids = -1, powers = 0, later = 0x7f7f;
        const auto fetch = [&](int s) __attribute__((always_inline)) {
            const int page = page_of(s + lane / kFewPages) + lane % kFewPages;
            ids = page < end ? pt[page] : -1;
            ids = ids < p.num_pages ? ids : -1;
            later = 0x7f7f;
            if (ids >= 0)
                later = *reinterpret_cast<const uint16_t *>(p.kv_scales + 2 * ((size_t)ids * p.Hkv + pc.g));
        };
        const auto load = [&](int s, typename Few::Kv8Regs &r) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < kFewPages; h++) {
                const int pid = __builtin_amdgcn_readlane(ids, kFewPages * (s % kSteps) + h);
                const size_t block = (size_t)max(pid, 0) * p.Hkv + pc.g;
                const int bytes = pid >= 0 ? kPageBytes : 0;   // (no records: zeros)
                const block_rsrc_t rk = block_rsrc(reinterpret_cast<const char *>(p.k_pages) + block * kPageBytes, bytes);
                const block_rsrc_t rv = block_rsrc(reinterpret_cast<const char *>(p.v_pages) + block * kPageBytes, bytes);
#pragma unroll
                for (int e = 0; e < D / 64; e++)
                    r.k[h][e] = ld_block16(rk, n * D + 16 * kq + 64 * e);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    r.v[h][i].load(rv, (4 * kq + i) * D + VE * n);
            }
        };

        typename Few::State st;
        typename Few::Kv8Regs ring[kRing];
        const bool row_ok = n < rows;
        const int token = pc.m * p.TT + (row_ok ? n / p.G : 0), head = pc.g * p.G + (row_ok ? n % p.G : 0);
        const uint16_t *qr = p.q + (int64_t)(sq.row0 + token) * p.q_stride + (int64_t)head * D;
        if (own > 0)
            fetch(0);
        u32x4_t qf[kKSteps / 2];
#pragma unroll
        for (int ks = 0; ks < kKSteps / 2; ks++)
            qf[ks] = row_ok ? *reinterpret_cast<const u32x4_t *>(qr + Few::q_dim(kq, ks)) : u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < kRing - 1; i++)
            if (i < own)
                load(i, ring[i]);
#pragma unroll
        for (int ks = 0; ks < kKSteps / 2; ks++)
            st.qf[0][ks] = __builtin_bit_cast(uint4, qf[ks] ^ p.q_sign);
        powers = later;
        const int full_end = min(first_lim, seg_end);
        st.lim[0] = min(row_ok ? sq.L - sq.c.Q + token + 1 : sq.L, seg_end);
        st.m_ref[0] = -INFINITY;
        st.lacc[0] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int jj = 0; jj < VE; jj++)
            st.acc[0][jj] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        for (int s0 = 0; s0 < own; s0 += kRing) {
#pragma unroll
            for (int i = 0; i < kRing; i++) {
                const int s = s0 + i, next = s + kRing - 1;
                if (s < own) {
                    if (s > 0 && s % kSteps == 0)
                        powers = later;
                    if (next < own) {
                        if (next % kSteps == 0)
                            fetch(next);
                        load(next, ring[(i + kRing - 1) % kRing]);
                    }
#pragma unroll
                    for (int h = 0; h < kFewPages; h++)
                        ring[i].power[h] = __builtin_amdgcn_readlane(powers, kFewPages * (s % kSteps) + h);
                    Few::page_step(p, st, ring[i], page_of(s), full_end, seg_end, kq);
                }
            }
        }

        // Sums and statistics of each wavefront, then a thread for four values of a row.
        constexpr int kParts = VE / 4;
        f32x4_t *const sums = reinterpret_cast<f32x4_t *>(lds);   // [wave][4][kParts][lane]
        float *const stats = reinterpret_cast<float *>(lds + kCodes);   // [wave][2][16]
        static_assert(kChunkWaves * 4 * kParts * kWave * 16 <= kCodes, "sums in front of the codes");
        lds_barrier();   // nobody reads the piece in front of this one any more
#pragma unroll
        for (int i = 0; i < 4; i++) {
#pragma unroll
            for (int e = 0; e < kParts; e++)
                sums[((wave * 4 + i) * kParts + e) * kWave + lane] =
                    f32x4_t{st.acc[0][4 * e][i], st.acc[0][4 * e + 1][i], st.acc[0][4 * e + 2][i], st.acc[0][4 * e + 3][i]};
            if (n == 0)
                stats[32 * wave + 16 + 4 * kq + i] = st.lacc[0][i];
        }
        if (kq == 0)
            stats[32 * wave + n] = st.m_ref[0];
        lds_barrier();
        const int tid = wave * kWave + lane, part = tid & 15, e = (tid >> 4) % kParts, r = tid / (16 * kParts);
        if (r < rows) {   // (of 16 or 32)
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int k = 0; k < kChunkWaves; k++)
                m = fmaxf(m, stats[32 * k + r]);
            f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < kChunkWaves; k++) {
                const float mk = stats[32 * k + r];
                const float f = mk == -INFINITY ? 0.0f : fast_exp2(mk - m);
                l += f * stats[32 * k + 16 + r];
                x += f * sums[((k * 4 + (r & 3)) * kParts + e) * kWave + 16 * (r >> 2) + part];
            }
            const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // NaN stays
            x *= inv;
            const int dim = VE * part + 4 * e;
            if (pc.whole) {
                uint16_t *dst = p.out + (int64_t)(sq.row0 + pc.m * p.TT + r / p.G) * p.out_stride + (int64_t)(pc.g * p.G + r % p.G) * D + dim;
                *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
            } else {
                const int64_t row = (int64_t)slot * kTileRows + r;
                *reinterpret_cast<f32x4_t *>(p.ws_o + row * D + dim) = x;
                if (part == 0 && e == 0)
                    p.ws_lse[row] = l == 0.0f ? -INFINITY : l > 0.0f ? m + __log2f(l) : l;
            }
        }
        lds_barrier();
    }

    // A worker's range.  A row's query is read by the workers of its row tile
    // alone, and output is written after it: by the one that has the whole tile,
    // or by the merge kernel (so the output may take the queries' place).
    // While a piece's result is written, the first tiles of the next one are already on
    // their way (few_rows starts and ends by itself).
    __device__ __forceinline__ static void work(const ChunkParams &p, const uint64_t *s_end, int w, int64_t begin, int64_t end, char *lds) {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = first_lane_int(threadIdx.x / kWave);
        const int h = lane >> 5;
        const int r = wave * kRowBlock + (lane & 31);
        if (begin >= end)
            return;
        Piece pc = locate_tile<k8>(p, s_end, begin, end);
        int64_t x = pc.next;
        if (threadIdx.x == 0) {
            const SeqInfo sq = seq_info<k8>(p, pc.b);
            const int at = pc.m * p.TT;
            p.cuts[w] = Cut{(int64_t)s_end[p.B - 1] * p.Hkv, pc.us, pc.n, pc.weight, sq.row0 + at, min(p.TT, sq.c.Q - at), pc.g * p.G};
        }
        if (pc.j0 >= pc.j1 && !next_piece<k8>(p, s_end, x, end, pc))
            return;
        bool first = pc.us <= begin;   // the range starts inside it: its partial result's slot
        State st;
        set_addresses(st, lds, wave, lane);
        // Queries of a piece: before its first tiles, and before the results of the
        // piece in front of it, since loads and stores finish in order.
        const auto queries = [&](const Piece &of) __attribute__((always_inline)) {
            const SeqInfo sq = seq_info<k8>(p, of.b);
            const int token = of.m * p.TT + r / p.G;
            const bool row_ok = r < p.TT * p.G && token < sq.c.Q;
            const int head = of.g * p.G + r % p.G;
            const uint16_t *qr = p.q + (int64_t)(sq.row0 + (row_ok ? token : 0)) * p.q_stride + (int64_t)(row_ok ? head : 0) * D + 8 * h;
#pragma unroll
            for (int ks = 0; ks < kKSteps; ks++)
                st.qf[ks] = row_ok ? *reinterpret_cast<const u32x4_t *>(qr + 16 * ks) : u32x4_t{0u, 0u, 0u, 0u};
        };
        bool few = is_few(p, pc);
        TilePages pages;
        if (!few) {
            queries(pc);
            pages = start(p, st, pc, lds, wave, lane);
        }
        for (;;) {
            if constexpr (k8) {
                if (few) {
                    few_rows(p, pc, first ? 2 * w : 2 * w + 1, lds, wave, lane);
                    if (!next_piece<k8>(p, s_end, x, end, pc))
                        return;
                    first = false;
                    few = is_few(p, pc);
                    if (!few) {
                        queries(pc);
                        pages = start(p, st, pc, lds, wave, lane);
                    } else {   // (nothing to keep meanwhile)
#pragma unroll
                        for (int ks = 0; ks < kKSteps; ks++)
                            st.qf[ks] = u32x4_t{0u, 0u, 0u, 0u};
                        pages = {};
                    }
                    continue;
                }
            }
            const SeqInfo sq = seq_info<k8>(p, pc.b);
            const int token = pc.m * p.TT + r / p.G;
            const bool row_ok = r < p.TT * p.G && token < sq.c.Q;
            const int head = pc.g * p.G + r % p.G;
            // the first row of the unit sees the fewest keys; tiles before
            // `plain` are seen whole by every row, and lie inside the context
            const int all_lim = sq.L - sq.c.Q + pc.m * p.TT + 1;
            const int plain = first_lane_int(min(max(max(all_lim, 0) / kKeyTile, pc.j0), pc.j1));
            st.lim = row_ok ? sq.L - sq.c.Q + token + 1 : 0;
            st.m_ref = kLowest;
            st.l = 0.0f;
#pragma unroll
            for (int ks = 0; ks < kKSteps; ks++)
                st.qf[ks] ^= p.q_sign;
#pragma unroll
            for (int dt = 0; dt < kDTiles; dt++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    st.o[dt][e] = 0.0f;
            // Tile i is used by two steps: its keys by step i - 1, its values by
            // step i.  After the barrier in front of step i tile i + 1 is there,
            // and nobody reads tile i - 1 any more, whose stage is filled next.
            const int n = pc.j1 - pc.j0, n_plain = plain - pc.j0;
            bool odd = false;
            const auto arrive = [&](int i, int later) __attribute__((always_inline)) {
                dma_wait<kLoads>(later);
                if (i >= n_plain && wave >= kTilePages)
                    odd |= clean_page(lds + i % kStages * kStage, wave, lane, sq.L - ((pc.j0 + i) * kTilePages + wave % kTilePages) * kPage);
                lds_barrier();
            };
            // Codes: tile i becomes bf16 once it is there, and its place is loaded
            // with tile i + 4.  A wavefront reads only codes that it loaded.
            const auto convert = [&](int i) __attribute__((always_inline)) {
                if constexpr (k8) {
                    if (i >= n)
                        return;
                    dma_wait<kLoads>(min(n - 1 - i, kCodeStages - 1));
                    char *codes = lds + kCodes + i % kCodeStages * kCodeBytes;
                    if (__builtin_expect(i % kWave == 0 && i > 0, 0))
                        pages.bytes = pages.later;
                    odd |= convert_page(st, codes + wave * kPageBytes, i % kStages, pages.power(i), i >= n_plain && wave >= kTilePages,
                                        sq.L - ((pc.j0 + i) * kTilePages + wave % kTilePages) * kPage, wave, lane);
                    const int next = i + kCodeStages;
                    if (next < n) {
                        if (__builtin_expect(next % kWave == 0, 0))
                            pages.fetch(p, next, pc.g, wave, lane);
                        dma_page(p, st, pages.id(next), pages.once, pc.g, codes, wave, lane);
                    }
                }
            };
            // Step i reads the keys of tile i + 1 and the values of tile i.  Meanwhile the
            // keys' wavefronts convert tile i + 2, before their own part of the step, and
            // the values' tile i + 1, after it: a SIMD has one of each, so its matrix
            // unit is not left alone.
            const auto before = [&](int i) __attribute__((always_inline)) {
                if (wave < kTilePages)
                    convert(i + 2);
            };
            const auto after = [&](int i) __attribute__((always_inline)) {
                if (wave >= kTilePages)
                    convert(i + 1);
                lds_barrier();
            };
            const auto room = [&](int i) { return st.lim - (pc.j0 + i) * kKeyTile - 4 * h; };
            const auto advance = [&](int i) __attribute__((always_inline)) {
                if constexpr (k8) {
                    before(i);
                } else {
                    arrive(i + 1, min(n - 2 - i, 1));
                    if (i + kStages - 1 < n)
                        dma_page(p, st, pages.next(i + kStages - 1), pages.once, pc.g, lds + (i + kStages - 1) % kStages * kStage, wave, lane);
                }
            };
            const auto step = [&](int i, Scores &c, Scores &next) __attribute__((always_inline)) {
                advance(i);
                tile_step<true>(p, st, c, next, i % kStages * kStage, (i + 1) % kStages * kStage, i >= n_plain, room(i));
                if constexpr (k8)
                    after(i);
            };
            if constexpr (k8) {
                convert(0);
                before(-1);
                lds_barrier();
            } else {
                arrive(0, min(n - 1, 2));
            }
            if (__any(row_ok)) {
                Scores a, b;
                scores(st, 0, a);
                if (k8 && n > 2)
                    lds_barrier();   // step 0 replaces the first keys
                largest(p, a);
                for (int i = 0; i + 1 < n; i += 2) {
                    step(i, a, b);
                    if (i + 2 >= n) {
                        a = b;
                        break;
                    }
                    step(i + 1, b, a);
                }
                tile_step<false>(p, st, a, b, (n - 1) % kStages * kStage, 0, n > n_plain, room(n - 1));
            } else {   // no row of this wavefront has a token: it only loads
                if (k8 && n > 2)
                    lds_barrier();
                for (int i = 0; i + 1 < n; i++) {
                    advance(i);
                    if constexpr (k8)
                        after(i);
                }
            }
            lds_barrier();
            if (n_plain < n) {   // the same for every wavefront
                // the stage that start() leaves alone (of codes, the values of the second
                // tile, which are converted after a barrier)
                int *flags = reinterpret_cast<int *>(lds + (kStages - 1) * kStage + (k8 ? kKBytes : 0));
                const bool mine = __any(odd);
                if (lane == 0)
                    flags[wave] = mine;
                lds_barrier();
                bool any = false;
#pragma unroll
                for (int i = 0; i < kChunkWaves; i++)
                    any |= flags[i] != 0;
                if (any)
                    add_odd(p, st, p.page_table + (size_t)pc.b * p.max_pages, pc.g, plain * kKeyTile, min(pc.j1 * kKeyTile, sq.L), h);
            }
            Piece nx = pc;
            const bool more = next_piece<k8>(p, s_end, x, end, nx);
            few = more && is_few(p, nx);
            if (more && !few) {
                queries(nx);
                pages = start(p, st, nx, lds, wave, lane);
            }
            if (row_ok)
                write_rows(p, st, sq, pc, first ? 2 * w : 2 * w + 1, r, token, head, h);
            if (!more)
                return;
            pc = nx;
            first = false;
        }
    }

    __device__ __forceinline__ static void write_rows(const ChunkParams &p, const State &st, const SeqInfo &sq, const Piece &pc, int slot, int r,
                                      int token, int head, int h) {
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

template <int D, bool k8>
__global__ __launch_bounds__(kChunkWaves * kWave, 2) void chunk_attn_kernel(ChunkParams p) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];   // the tiles, then the prefix
    uint64_t *s_tiles = reinterpret_cast<uint64_t *>(lds + Chunk<D, k8>::kLds);
    tile_ends<k8>(p, s_tiles);
    const int64_t ptot = first_lane_int64((int64_t)s_tiles[p.B - 1]) * p.Hkv;
    const int w = xcd_worker(blockIdx.x, p.W);
    const int64_t begin = first_lane_int64(range_start(ptot, w, p.W, p.range_inv));
    const int64_t end = first_lane_int64(range_start(ptot, w + 1, p.W, p.range_inv));
    if (ptot == 0 && w == p.W - 1 && threadIdx.x == 0)
        p.cuts[w].ptot = 0;
    Chunk<D, k8>::work(p, s_tiles, w, begin, end, lds);
}

// Joins the pieces of the units that a worker boundary cuts: workgroup x takes
// the unit that boundary x + 1 falls into, if it is the first one inside it;
// workgroups along y take merge_rows(D) rows each, D / 8 lanes per row.  The
// loads of several pieces are under way at once: one after the other, sixteen
// pieces took 21 us.
constexpr int kMergeThreads = 256, kMergeAhead = 4;
constexpr int merge_rows(int D) { return kMergeThreads / (D / 8); }

template <int D>
__global__ __launch_bounds__(kMergeThreads) void chunk_merge_kernel(ChunkParams p) {
    constexpr int kMergeRows = merge_rows(D), kMergeLanes = D / 8;
    const int w = blockIdx.x + 1;
    Cut cut = p.cuts[w];
    const int64_t ptot = p.cuts[p.W - 1].ptot;   // (that range is never empty)
    if (ptot == 0)
        return;
    const int64_t x = range_start(ptot, w, p.W, p.range_inv);
    const int64_t prev = range_start(ptot, w - 1, p.W, p.range_inv);
    if (x >= ptot || x == prev)
        return;
    if (ptot < p.W)   // some ranges are empty, w's maybe
        cut = p.cuts[worker_of(ptot, x, p.W)];
    if (x == cut.us || tile_at(x - cut.us, cut.weight) >= cut.n || prev > cut.us)
        return;   // no tiles are cut off here, or an earlier boundary cuts the unit too
    const int places = cut.n * cut.weight;
    const UnitSplit u = unit_split(ptot, cut.us, places, p.W);
    constexpr int kPer = D / kMergeLanes;
    const int r = blockIdx.y * kMergeRows + threadIdx.x / kMergeLanes, part = threadIdx.x % kMergeLanes;
    const bool row_ok = r < cut.tokens * p.G;   // (of whole rows of lanes)
    if (blockIdx.y * kMergeRows >= cut.tokens * p.G)
        return;
    __shared__ int s_slot[kMergeThreads];   // slots of up to 256 parts, -1: no tile starts among its places
    float M = kLowest, sum = 0.0f, o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; e++)
        o[e] = 0.0f;
    for (int base = 0; base < u.nparts; base += kMergeThreads) {
        const int n = min(u.nparts - base, kMergeThreads);
        __syncthreads();
        if ((int)threadIdx.x < n) {
            const int k = base + threadIdx.x;
            const int64_t lo = u.dense ? max(range_start(ptot, u.wlo + k, p.W, p.range_inv) - cut.us, (int64_t)0) : k;
            const int64_t hi = u.dense ? min(range_start(ptot, u.wlo + k + 1, p.W, p.range_inv) - cut.us, (int64_t)places) : k + 1;
            s_slot[threadIdx.x] = tile_at(lo, cut.weight) < tile_at(hi, cut.weight) ? u.slot(k) : -1;
        }
        __syncthreads();
        if (!row_ok)
            continue;
        for (int k0 = 0; k0 < n; k0 += kMergeAhead) {
            f32x4_t v[kMergeAhead][kPer / 4];
            float lse[kMergeAhead];
#pragma unroll
            for (int i = 0; i < kMergeAhead; i++) {
                const int slot = s_slot[min(k0 + i, n - 1)];
                const int64_t row = (int64_t)max(slot, 0) * kTileRows + r;
                lse[i] = slot < 0 || k0 + i >= n ? -INFINITY : p.ws_lse[row];
#pragma unroll
                for (int e = 0; e < kPer / 4; e++)
                    v[i][e] = *reinterpret_cast<const f32x4_t *>(p.ws_o + row * D + kPer * part + 4 * e);
            }
            float m = M;
#pragma unroll
            for (int i = 0; i < kMergeAhead; i++)
                m = fmaxf(m, lse[i]);
            const float scale = fmaxf(fast_exp2(M - m), kTiny);   // (an infinite piece stays infinite)
            M = m;
            sum *= scale;
#pragma unroll
            for (int e = 0; e < kPer; e++)
                o[e] *= scale;
#pragma unroll
            for (int i = 0; i < kMergeAhead; i++) {
                if (lse[i] == -INFINITY)   // no piece, or one without a visible key
                    continue;
                const float a = fmaxf(fast_exp2(lse[i] - M), kTiny);
                sum += a;
#pragma unroll
                for (int e = 0; e < kPer; e++)
                    o[e] += a * v[i][e / 4][e % 4];
            }
        }
    }
    if (!row_ok)
        return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t *dst = p.out + (int64_t)(cut.row + r / p.G) * p.out_stride + (int64_t)(cut.head + r % p.G) * D + kPer * part;
#pragma unroll
    for (int e = 0; e < kPer; e += 4)
        *reinterpret_cast<uint2 *>(dst + e) =
            make_uint2(pack_bf16x2(o[e] * inv, o[e + 1] * inv), pack_bf16x2(o[e + 2] * inv, o[e + 3] * inv));
}

struct ChunkPlan {
    int G, TT, W;
    size_t ws_lse_off, ws_cut_off, ws_bytes;
};

int make_chunk_plan(const ts_chunk_shape *s, bool k8, ChunkPlan *pl) {
    const int st = check_chunk_shape(s);
    if (st)
        return st;
    pl->G = s->num_q_heads / s->num_kv_heads;
    pl->TT = kTileRows / pl->G;
    // KV tiles of the call, from above
    const int64_t tiles = ((int64_t)s->num_tokens / pl->TT + std::min(s->num_seqs, s->num_tokens)) * s->num_kv_heads *
                          (((int64_t)s->max_ctx_len + kKeyTile - 1) / kKeyTile);
    const int64_t most = workers_bound(places_bound(s->num_seqs, s->num_kv_heads, s->num_tokens, pl->TT,
                                                    (int64_t)s->max_pages_per_seq * kPage, k8));
    if (s->num_workers > most)
        return fail(TS_ERR_SHAPE, "num_workers %d exceeds %lld, what this shape's work can be cut into", s->num_workers,
                    (long long)most);
    pl->W = s->num_workers > 0 ? s->num_workers : (int)std::max<int64_t>(1, std::min({(int64_t)256, tiles / 2, most}));
    const size_t rows = 2 * (size_t)pl->W * kTileRows;
    pl->ws_lse_off = rows * s->head_dim * sizeof(float);
    pl->ws_cut_off = pl->ws_lse_off + rows * sizeof(float);
    pl->ws_bytes = (pl->ws_cut_off + pl->W * sizeof(Cut) + 255) & ~(size_t)255;
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

// ts_chunk_attn and ts_chunk_attn_kv8.
template <bool k8>
static int launch_chunk(const ts_chunk_shape *s, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                        const void *kv_scales, const int32_t *page_table, const int32_t *ctx_lens,
                        const int32_t *q_starts, void *out, int64_t out_stride, float scale, void *workspace,
                        size_t workspace_bytes, void *stream) {
    clear_error();
    ChunkPlan pl;
    int st = make_chunk_plan(s, k8, &pl);
    if (st)
        return st;
    if (s->num_tokens == 0)
        return TS_OK;   // no rows, whose tensors may be NULL
    if (!q || !k_pages || !v_pages || !page_table || !ctx_lens || !q_starts || !out || !workspace)
        return fail(TS_ERR_NULL, "a pointer is NULL");
    if (k8 && !kv_scales)
        return fail(TS_ERR_NULL, "kv_scales is NULL");
    if (!std::isfinite(scale))
        return fail(TS_ERR_ARG, "scale must be finite");
    if (workspace_bytes < pl.ws_bytes)
        return fail(TS_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, pl.ws_bytes);
    if ((((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)out | (uintptr_t)kv_scales) & 15) || ((uintptr_t)workspace & 255))
        return fail(TS_ERR_ARG, "misaligned pointer (tensors 16 B, workspace 256 B)");
    const int64_t row = (int64_t)s->num_q_heads * s->head_dim;
    if ((st = check_stride("q_stride", q_stride, row)) || (st = check_stride("out_stride", out_stride, row)))
        return st;
    if (out == q && out_stride != q_stride)
        return fail(TS_ERR_ARG, "out == q needs equal strides");
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
    p.cuts = reinterpret_cast<Cut *>(static_cast<char *>(workspace) + pl.ws_cut_off);
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
    // (a scale of 0 leaves equal scores, but no product of it with the -inf of a
    // masked one)
    p.scale_log2 = std::max(std::fabs(scale) * 1.44269504088896341f, 1e-30f);
    p.q_sign = std::signbit(scale) ? 0x80008000u : 0u;
    p.kv_scales = static_cast<const uint8_t *>(kv_scales);
    const size_t pre = (size_t)s->num_seqs * sizeof(uint64_t);
    const bool small = s->head_dim == 64;
    const auto main_k = small ? chunk_attn_kernel<64, k8> : chunk_attn_kernel<128, k8>;
    const auto merge_k = small ? chunk_merge_kernel<64> : chunk_merge_kernel<128>;
    hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(main_k, dim3((unsigned)pl.W), dim3(kChunkWaves * kWave),
                       pre + (small ? Chunk<64, k8>::kLds : Chunk<128, k8>::kLds), hs, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return hip_fail(e, "chunk attention launch");
    if (pl.W > 1) {
        hipLaunchKernelGGL(merge_k, dim3((unsigned)pl.W - 1, kTileRows / merge_rows(s->head_dim)), dim3(kMergeThreads),
                           0, hs, p);
        if ((e = hipGetLastError()) != hipSuccess)
            return hip_fail(e, "chunk merge launch");
    }
    return TS_OK;
}

}  // namespace tsattn

using namespace tsattn;

extern "C" {

size_t ts_chunk_attn_workspace_size(const ts_chunk_shape *s) {
    clear_error();
    ChunkPlan pl;
    return make_chunk_plan(s, false, &pl) == TS_OK ? pl.ws_bytes : 0;
}

size_t ts_chunk_attn_kv8_workspace_size(const ts_chunk_shape *s) {
    clear_error();
    ChunkPlan pl;
    return make_chunk_plan(s, true, &pl) == TS_OK ? pl.ws_bytes : 0;
}

int ts_chunk_attn(const ts_chunk_shape *s, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                  const int32_t *page_table, const int32_t *ctx_lens, const int32_t *q_starts, void *out,
                  int64_t out_stride, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    return launch_chunk<false>(s, q, q_stride, k_pages, v_pages, nullptr, page_table, ctx_lens, q_starts, out, out_stride,
                               scale, workspace, workspace_bytes, stream);
}

int ts_chunk_attn_kv8(const ts_chunk_shape *s, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages,
                      const void *kv_scales, const int32_t *page_table, const int32_t *ctx_lens,
                      const int32_t *q_starts, void *out, int64_t out_stride, float scale, void *workspace,
                      size_t workspace_bytes, void *stream) {
    return launch_chunk<true>(s, q, q_stride, k_pages, v_pages, kv_scales, page_table, ctx_lens, q_starts, out,
                              out_stride, scale, workspace, workspace_bytes, stream);
}

}  // extern "C"
