// rope_append.hip -- head norms of the queries and keys, position rotation and
// the append to the paged cache, in one pass over the projections' output.
//
// For a packed row of sequence b at position p = L_b - Q_b + i, and one head's
// vector x (head_dim values):
//   norm      x <- x * w / sqrt(mean(x^2) + eps)            (if w is given)
//   rotation  pairs (x_j, x_{j + rot/2}), or (x_{2j}, x_{2j+1}) interleaved,
//             turn by the angle p * inv_freq[j], j < rot/2; dimensions from rot
//             on are kept.
// Queries go to q_out, keys and values into their page.  Everything is held in
// float32 between the bf16 inputs and the one rounding at the end.  The angle
// is formed in float64 in turns, reduced to half a turn there and only then
// rounded: at position 10^6 a float32 angle would be off by 0.06 rad.
//
// What bounds it: each vector is read once and written once, so memory; the
// chain of small loads in front of a row's first store (its sequence, lengths
// and page) where there are few rows.  So one workgroup takes one row: its
// first wavefront runs that chain and the row's rot/2 angles (one per lane)
// while the loads of all wavefronts' heads, which do not depend on it, are in
// flight; angles and page reach the others through LDS.  A head is held by
// head_dim / 8 lanes with 16 bytes each, so the sum of a norm is four lane
// moves, and the partner of a half-split pair is one lane exchange of the
// packed values away.
// Measured, 32/8 heads of 128: 8,192 rows with norms 38 us, 5.3 TB/s read and
// written (the rate of a large copy: 4.9); 8 rows 4.5 us.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>

#include "attn_common.h"
#include "chunk_common.h"
#include "ts_attn.h"
#include "ts_internal.h"

namespace tsattn {

namespace {

constexpr int kRopeWaves = 4;
constexpr int kRopePasses = 3;   // head groups of a wavefront whose loads are in flight together

struct RopeParams {
    const uint16_t *q, *k, *v;       // rows of q_stride / k_stride / v_stride elements
    uint16_t *q_out;
    uint16_t *k_pages, *v_pages;     // [num_pages][Hkv][16][D]
    const int32_t *page_table, *ctx_lens, *q_starts;
    const float *inv_freq;
    const uint16_t *q_norm, *k_norm; // [D] or NULL
    int64_t q_stride, k_stride, v_stride, q_out_stride, num_pages;
    int B, Hq, Hkv, max_pages, rot, interleaved, num_tokens;
    float eps;
};

// What the first wavefront finds out about a row.
struct RowInfo {
    float cos[64], sin[64];   // of pair j
    int64_t slot;             // (page * Hkv * 16 + position % 16), or -1: no place in the pool
    int used;                 // the row belongs to a sequence
};

__device__ __forceinline__ void unpack8(u32x4_t u, float x[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[2 * i] = bf16_lo(u[i]);
        x[2 * i + 1] = bf16_hi(u[i]);
    }
}
__device__ __forceinline__ u32x4_t pack8(const float x[8]) {
    u32x4_t u;
#pragma unroll
    for (int i = 0; i < 4; i++)
        u[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    return u;
}

constexpr int kDppMirror = 0x140;   // lane i <-> 15 - i within 16
template <int kLanes>
__device__ __forceinline__ float sum_head(float x) {
    x = sum8(x);
    if constexpr (kLanes == 16)
        x += dpp_f32<kDppMirror>(x);
    return x;
}

template <int D>
__global__ __launch_bounds__(kRopeWaves * kWave) void rope_append_kernel(RopeParams p) {
    constexpr int kLanes = D / 8;            // lanes per head
    constexpr int kHeads = kWave / kLanes;   // heads per wavefront and pass
    __shared__ RowInfo info;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = first_lane_int(threadIdx.x / kWave);
    const int64_t t = blockIdx.x;
    const int c = lane % kLanes;             // 16-byte piece of the head
    const int heads = p.Hq + 2 * p.Hkv;
    const int half = p.rot / 2;

    for (int base = 0; base < heads; base += kRopePasses * kRopeWaves * kHeads) {
        u32x4_t raw[kRopePasses];
#pragma unroll
        for (int i = 0; i < kRopePasses; i++) {
            const int h = base + (i * kRopeWaves + wave) * kHeads + lane / kLanes;
            const uint16_t *src = h < p.Hq            ? p.q + t * p.q_stride + (int64_t)h * D
                                  : h < p.Hq + p.Hkv ? p.k + t * p.k_stride + (int64_t)(h - p.Hq) * D
                                                      : p.v + t * p.v_stride + (int64_t)(h - p.Hq - p.Hkv) * D;
            raw[i] = h < heads ? *reinterpret_cast<const u32x4_t *>(src + 8 * c) : u32x4_t{0u, 0u, 0u, 0u};
        }
        if (base == 0) {
            if (wave == 0) {
                const int b = find_packed_seq(p.q_starts, p.B, (int)t);
                const int first = ld_meta(p.q_starts, b), end = min(ld_meta(p.q_starts, b + 1), p.num_tokens);
                const int64_t pos = clamped_len(ld_meta(p.ctx_lens, b), p.max_pages) - (end - t);
                const bool used = first <= t && t < end;
                int64_t slot = -1;
                if (used && pos >= 0) {   // (below the clamped length, so inside the table)
                    const int page = ld_meta(p.page_table, (size_t)b * p.max_pages + pos / kPage);
                    if (page >= 0 && page < p.num_pages)
                        slot = (int64_t)page * p.Hkv * kPage + pos % kPage;
                }
                if (lane < half) {
                    const double turns = (double)pos * (double)p.inv_freq[lane] * 0.15915494309189533577;   // 1 / 2 pi
                    float s, co;
                    sincospif((float)(2.0 * (turns - rint(turns))), &s, &co);
                    info.cos[lane] = co;
                    info.sin[lane] = s;
                }
                if (lane == 0) {
                    info.slot = slot;
                    info.used = used;
                }
            }
            __syncthreads();
            if (!info.used)
                return;   // behind the last sequence
        }
        const int64_t slot = info.slot;
#pragma unroll
        for (int i = 0; i < kRopePasses; i++) {
            const int h = base + (i * kRopeWaves + wave) * kHeads + lane / kLanes;
            const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
            u32x4_t y = raw[i];
            // (whole wavefronts of values skip the arithmetic)
            if (base + (i * kRopeWaves + wave) * kHeads < p.Hq + p.Hkv) {
                // the partner piece of a half-split pair, in the same head
                const int pieces = p.rot / 16;   // pieces of each half
                const int other = p.interleaved ? c : c < pieces ? c + pieces : c < 2 * pieces ? c - pieces : c;
                u32x4_t raw2;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    raw2[e] = __shfl(raw[i][e], lane - c + other, kWave);
                float x[8], z[8];
                unpack8(raw[i], x);
                unpack8(raw2, z);
                const uint16_t *w = is_q ? p.q_norm : p.k_norm;
                // one wavefront can hold queries without a norm and keys with
                // one: every lane takes part in the sum
                if (p.q_norm || p.k_norm) {
                    float ss = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        ss += x[e] * x[e];
                    ss = sum_head<kLanes>(ss);
                    if (w && !is_v) {
                        const float r = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
                        float wx[8], wz[8];
                        unpack8(*reinterpret_cast<const u32x4_t *>(w + 8 * c), wx);
                        unpack8(*reinterpret_cast<const u32x4_t *>(w + 8 * other), wz);
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            x[e] *= r * wx[e];
                            z[e] *= r * wz[e];
                        }
                    }
                }
                if (8 * c < p.rot) {
                    if (p.interleaved) {
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const float co = info.cos[4 * c + e], s = info.sin[4 * c + e];
                            const float a = x[2 * e], d = x[2 * e + 1];
                            x[2 * e] = a * co - d * s;
                            x[2 * e + 1] = d * co + a * s;
                        }
                    } else {
                        const int j = 8 * (c < pieces ? c : c - pieces);
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            const float co = info.cos[j + e], s = info.sin[j + e];
                            x[e] = c < pieces ? x[e] * co - z[e] * s : x[e] * co + z[e] * s;
                        }
                    }
                }
                if (!is_v)
                    y = pack8(x);
            }
            if (h >= heads)
                continue;
            if (is_q) {
                *reinterpret_cast<u32x4_t *>(p.q_out + t * p.q_out_stride + (int64_t)h * D + 8 * c) = y;
            } else if (slot >= 0) {
                const int g = h - p.Hq - (is_v ? p.Hkv : 0);
                *reinterpret_cast<u32x4_t *>((is_v ? p.v_pages : p.k_pages) + (slot + (int64_t)g * kPage) * D + 8 * c) = y;
            }
        }
    }
}

}  // namespace

}  // namespace tsattn

using namespace tsattn;

extern "C" {

int ts_rope_append(const ts_chunk_shape *s, const ts_rope_config *cfg, const void *q, const void *k, const void *v,
                   void *q_out, void *k_pages, void *v_pages, const int32_t *page_table, const int32_t *ctx_lens,
                   const int32_t *q_starts, const float *inv_freq, const void *q_norm, const void *k_norm,
                   void *stream) {
    clear_error();
    int st = check_chunk_shape(s);
    if (st)
        return st;
    if (s->num_tokens == 0)
        return TS_OK;   // no rows, whose tensors may be NULL
    if (!cfg || !q || !k || !v || !q_out || !k_pages || !v_pages || !page_table || !ctx_lens || !q_starts)
        return fail(TS_ERR_NULL, "a pointer is NULL");
    const int D = s->head_dim;
    if (cfg->rot_dim < 0 || cfg->rot_dim > D || cfg->rot_dim % 16)
        return fail(TS_ERR_ARG, "rot_dim %d must be a multiple of 16 up to head_dim %d", cfg->rot_dim, D);
    if (cfg->rot_dim > 0 && !inv_freq)
        return fail(TS_ERR_NULL, "inv_freq is NULL");
    if (cfg->interleaved != 0 && cfg->interleaved != 1)
        return fail(TS_ERR_ARG, "interleaved %d must be 0 or 1", cfg->interleaved);
    if (cfg->reserved != 0)
        return fail(TS_ERR_ARG, "reserved must be 0");
    if ((q_norm || k_norm) && !(cfg->eps >= 0.0f && std::isfinite(cfg->eps)))
        return fail(TS_ERR_ARG, "eps must be finite and not negative");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)k_pages | (uintptr_t)v_pages |
         (uintptr_t)q_norm | (uintptr_t)k_norm) & 15)
        return fail(TS_ERR_ARG, "misaligned pointer (16 B needed)");
    const int64_t q_row = (int64_t)s->num_q_heads * D, kv_row = (int64_t)s->num_kv_heads * D;
    if ((st = check_stride("q_stride", cfg->q_stride, q_row)) || (st = check_stride("k_stride", cfg->k_stride, kv_row)) ||
        (st = check_stride("v_stride", cfg->v_stride, kv_row)) ||
        (st = check_stride("q_out_stride", cfg->q_out_stride, q_row)))
        return st;
    if (q_out == q && cfg->q_out_stride != cfg->q_stride)
        return fail(TS_ERR_ARG, "q_out == q needs equal strides");
    if ((st = check_device()))
        return st;
    RopeParams p;
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.q_out = static_cast<uint16_t *>(q_out);
    p.k_pages = static_cast<uint16_t *>(k_pages);
    p.v_pages = static_cast<uint16_t *>(v_pages);
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.q_starts = q_starts;
    p.inv_freq = inv_freq;
    p.q_norm = static_cast<const uint16_t *>(q_norm);
    p.k_norm = static_cast<const uint16_t *>(k_norm);
    p.q_stride = cfg->q_stride;
    p.k_stride = cfg->k_stride;
    p.v_stride = cfg->v_stride;
    p.q_out_stride = cfg->q_out_stride;
    p.num_pages = s->num_pages;
    p.B = s->num_seqs;
    p.Hq = s->num_q_heads;
    p.Hkv = s->num_kv_heads;
    p.max_pages = s->max_pages_per_seq;
    p.num_tokens = s->num_tokens;
    p.rot = cfg->rot_dim;
    p.interleaved = cfg->interleaved;
    p.eps = cfg->eps;
    const auto kernel = D == 64 ? rope_append_kernel<64> : rope_append_kernel<128>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)s->num_tokens), dim3(kRopeWaves * kWave), 0,
                       reinterpret_cast<hipStream_t>(stream), p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TS_OK : hip_fail(e, "rotation and append launch");
}

}  // extern "C"
