// rope_append_kv8.hip -- head norms, position rotation and the append to the
// cache held in 8 bits (kv8_common.h), in one pass.
//
// Norm and rotation are those of rope_append.hip, in float32.  A page and KV head
// then takes for its new tokens' keys (values alike), x in float32:
//   m = max |x| over them (finite values), 2^k the smallest power with
//   m <= 448 * 2^k; where the page holds tokens in front of the new ones, with
//   power 2^h, k becomes max(k, h) and their codes are scaled by 2^(h - k);
//   code = e4m3(x / 2^k).
// A key is thus rounded once, from float32.
//
// A page's power depends on all of its new tokens, so a workgroup takes a page of
// a sequence, for one KV head and its query heads: 16 slots x D / 8 lanes, 16
// bytes of a head each, so that the page's keys are one load of the workgroup and
// their maximum is a few lane moves and one exchange through LDS.  The slots of
// held tokens, which have no row, keep those tokens' codes.  Nothing is laid out
// in memory first: sequence b's pages are given the places from
// floor(q_starts[b] / 16) + 2 b on, which is room enough for any position of its
// rows, and a workgroup finds its sequence among those closed sums.
//
// What bounds it.  Many rows: vector instructions beside the bytes: 8,192 rows of 32/8
// heads with norms take 44.7 us for 185 MB (4.1 TB/s; a large copy of as many takes
// 38).  From 53: norm weights in one factor with the angles, and a conversion that
// divides by the power, 50; the order of pairs a constant of the kernel, and
// frequencies loaded with the rows instead of one by one behind them, 48.5; no guard
// around each row's load, and sines by a series that takes turns, 47; norm weights
// loaded with the rows 44.7.  Several KV heads to a workgroup, which find their
// sequence and angles once, took 56 (2), 64 (4) and 73 us (8) instead of 53: fewer
// loads are under way.  Bounds on registers for five wavefronts per SIMD instead of
// four: 49.2 instead of 48.5; for more: 74 and 117 (spills).  Few rows: the chain
// starts -> lengths -> rows -> maximum -> stores, 4.6 us for 8 of them in a graph.
#include <hip/hip_runtime.h>

#include "attn_common.h"
#include "chunk_common.h"
#include "kv8_common.h"
#include "rope_common.h"
#include "ts_attn.h"
#include "ts_internal.h"

namespace tsattn {

namespace {

struct Rope8Params {
    const uint16_t *q, *k, *v;       // rows of q_stride / k_stride / v_stride elements
    uint16_t *q_out;
    uint8_t *k_pages, *v_pages;      // [num_pages][Hkv][16][D]
    uint8_t *scales;                 // [num_pages][Hkv][2]
    const int32_t *page_table, *ctx_lens, *q_starts;
    const float *inv_freq;
    const uint16_t *q_norm, *k_norm; // [D] or NULL
    int64_t q_stride, k_stride, v_stride, q_out_stride, num_pages;
    int B, Hq, Hkv, G, max_pages, rot, num_tokens;
    float eps;
};

constexpr int kQueries = 4;   // query heads whose loads are in flight together

// The largest of eight sizes, as the bits of a float: those of infinite and NaN values
// are above every finite one's.
__device__ __forceinline__ uint32_t max_abs8(const float x[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++)
        m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    return m;
}
// Finite values alone.
__device__ __forceinline__ uint32_t max_finite8(const float x[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const uint32_t u = __float_as_uint(x[e]) & 0x7fffffffu;
        m = max(m, u < 0x7f800000u ? u : 0u);
    }
    return m;
}
// Of a wavefront.  (The bits of sizes compare as the sizes do, but for NaN.)
__device__ __forceinline__ uint32_t max_wave(uint32_t x) {
    const auto step = [&](int y) { x = max(x, (uint32_t)y); };
    step(__builtin_amdgcn_update_dpp(0, (int)x, kDppXor1, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, (int)x, kDppXor2, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, (int)x, kDppHalfMirror, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, (int)x, kDppMirror, 0xf, 0xf, true));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(h[0], h[1]);
}

// Sine and cosine of f turns, |f| <= 1/2: of the angle's distance from the nearest
// quarter, |x| <= pi / 4, by their series up to x^9 and x^8 (what follows is below
// 2^-28 and 2^-25), exchanged and signed by the quarter.
__device__ __forceinline__ void sincos_turns(float f, float *sine, float *cosine) {
    const float quarter = rintf(4.0f * f);
    const float x = fmaf(-0.25f, quarter, f) * 6.283185307179586f, z = x * x;   // (the difference is exact)
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 40320.0f, -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const int n = (int)quarter;
    const uint32_t a = __float_as_uint(n & 1 ? c : s), b = __float_as_uint(n & 1 ? s : c);
    *sine = __uint_as_float(a ^ ((uint32_t)n << 30 & 0x80000000u));
    *cosine = __uint_as_float(b ^ ((uint32_t)(n + 1) << 30 & 0x80000000u));
}

template <int D, bool kInterleaved>
__global__ __launch_bounds__(kPage * D / 8) void rope_append_kv8_kernel(Rope8Params p) {
    constexpr int kLanes = D / 8;                  // lanes per head
    constexpr int kWaves = kPage * kLanes / kWave;
    __shared__ uint32_t s_max[2][kWaves], s_finite[2][kWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int slot = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
    const int g = blockIdx.y, T = p.num_tokens;

    const auto start = [&](int b) { return min(max(p.q_starts[b], 0), T); };
    const auto place = [&](int b) { return start(b) / kPage + 2 * b; };
    const int b = count_before(p.B, [&](int i) { return place(i + 1) <= (int)blockIdx.x; });
    const int first = first_lane_int(start(b)), Q = first_lane_int(start(b + 1)) - first;
    const int L = clamped_len(ld_meta(p.ctx_lens, b), p.max_pages);
    const int P = L - Q;                           // the position of the first row
    const int at = (int)blockIdx.x - (first / kPage + 2 * b);
    const int page = (P >> 4) + at;                // (rounded down, also below 0)
    if (Q <= 0 || at < 0 || page * kPage >= L)
        return;
    const int pos = page * kPage + slot;
    const bool active = pos >= P && pos < L;
    const int64_t row = first + (active ? pos - P : 0);

    // This lane's pairs: (x_j, x_{j + rot / 2}) with the partner lane `other`, j =
    // 8 (c mod pieces) + e; interleaved, (x_{2 j}, x_{2 j + 1}), j = 4 c + e.  The
    // two lanes of a half-split pair work out four of the eight angles each.
    const int pieces = p.rot / 16;                 // pieces of each half
    const bool upper = !kInterleaved && c >= pieces;
    const int other = kInterleaved ? c : c < pieces ? c + pieces : c < 2 * pieces ? c - pieces : c;
    const bool turns_here = 8 * c < p.rot;

    // frequencies and rows, which do not depend on the page, then the page
    struct __attribute__((packed, aligned(4))) Freqs {
        float x[4];
    } freq = {};
    if (p.rot > 0) {
        const int j = kInterleaved ? 4 * c : upper ? 8 * (c - pieces) + 4 : 8 * c;
        freq = *reinterpret_cast<const Freqs *>(p.inv_freq + (turns_here ? j : 0));   // (rot is 16 or more)
    }
    struct Weights {
        u32x4_t own, partner;
    };
    const auto weights = [&](const uint16_t *w) {
        Weights r = {};
        if (w) {
            r.own = *reinterpret_cast<const u32x4_t *>(w + 8 * c);
            if constexpr (!kInterleaved)
                r.partner = *reinterpret_cast<const u32x4_t *>(w + 8 * other);
        }
        return r;
    };
    const Weights k_weights = weights(p.k_norm), q_weights = weights(p.q_norm);
    // (lanes without a row read the first one)
    const auto load = [&](const uint16_t *x, int64_t stride, int h) {
        return *reinterpret_cast<const u32x4_t *>(x + row * stride + (int64_t)h * D + 8 * c);
    };
    const u32x4_t raw_k = load(p.k, p.k_stride, g), raw_v = load(p.v, p.v_stride, g);
    u32x4_t raw_q[kQueries];
#pragma unroll
    for (int i = 0; i < kQueries; i++)
        raw_q[i] = load(p.q, p.q_stride, g * p.G + min(i, p.G - 1));
    int64_t block = -1;                            // the page's place in the pool
    if (page >= 0) {
        const int pid = ld_meta(p.page_table, (size_t)b * p.max_pages + page);
        if (pid >= 0 && pid < p.num_pages)
            block = (int64_t)pid * p.Hkv + g;
    }
    const int held = block >= 0 ? max(P - page * kPage, 0) : 0;   // tokens that the page holds already
    uint16_t *const power = reinterpret_cast<uint16_t *>(p.scales) + max(block, (int64_t)0);
    const int64_t code_at = (max(block, (int64_t)0) * kPage + slot) * D + 8 * c;
    int old = 0;
    u32x2_t old_k = {0u, 0u}, old_v = {0u, 0u};
    if (held > 0) {
        old = *power;
        if (slot < held) {
            old_k = *reinterpret_cast<const u32x2_t *>(p.k_pages + code_at);
            old_v = *reinterpret_cast<const u32x2_t *>(p.v_pages + code_at);
        }
    }

    float co[8], si[8];                            // interleaved: of pair e / 2
    const auto angles = [&]() __attribute__((always_inline)) {
        float mc[4], ms[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const double turns = (double)pos * (double)freq.x[e] * 0.15915494309189533577;   // 1 / 2 pi
            sincos_turns((float)(turns - rint(turns)), &ms[e], &mc[e]);
            mc[e] = turns_here ? mc[e] : 1.0f;
            ms[e] = turns_here ? ms[e] : 0.0f;
        }
        if (kInterleaved) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                co[e] = mc[e / 2];
                si[e] = e % 2 ? ms[e / 2] : -ms[e / 2];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float pc = __shfl(mc[e], lane - c + other, kWave), ps = __shfl(ms[e], lane - c + other, kWave);
                co[e] = upper ? pc : mc[e];
                si[e] = upper ? ps : -ms[e];
                co[e + 4] = upper ? mc[e] : pc;
                si[e + 4] = upper ? ms[e] : -ps;
            }
        }
    };
    // A head's value is r (x a + z b), z its partner in the pair and r its norm's
    // factor, with the norm's weights in a and b.
    const auto factors = [&](const uint16_t *w, const Weights &raw, float a[8], float b[8]) __attribute__((always_inline)) {
        float wx[8], wz[8];
        unpack8(raw.own, wx);
        unpack8(raw.partner, wz);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            a[e] = w ? wx[e] * co[e] : co[e];
            b[e] = w ? (kInterleaved ? wx[e ^ 1] : wz[e]) * si[e] : si[e];
        }
    };
    const auto turned = [&](u32x4_t raw, bool norm, const float a[8], const float b[8], float x[8]) __attribute__((always_inline)) {
        u32x4_t raw2;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            raw2[e] = kInterleaved ? raw[e] << 16 | raw[e] >> 16 : __shfl(raw[e], lane - c + other, kWave);
            raw2[e] = turns_here ? raw2[e] : 0;    // (an infinite value times a sine of zero)
        }
        float z[8];
        unpack8(raw, x);
        unpack8(raw2, z);
        float r = 1.0f;
        if (norm) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++)
                ss += x[e] * x[e];
            r = __builtin_amdgcn_rsqf(sum_head<kLanes>(ss) * (1.0f / D) + p.eps);
        }
#pragma unroll
        for (int e = 0; e < 8; e++)
            x[e] = (x[e] * a[e] + z[e] * b[e]) * r;
    };

    const bool busy = __any(active);               // this wavefront has a row
    float xk[8], a[8], f[8];
    if (busy) {
        angles();
        factors(p.k_norm, k_weights, a, f);
        turned(raw_k, p.k_norm, a, f, xk);
        float xv[8];
        unpack8(raw_v, xv);
        const uint32_t mk = max_wave(active ? max_abs8(xk) : 0), mv = max_wave(active ? max_abs8(xv) : 0);
        uint32_t fk = mk, fv = mv;
        if (__builtin_expect(max(mk, mv) >= 0x7f800000u, 0)) {
            fk = max_wave(active ? max_finite8(xk) : 0);
            fv = max_wave(active ? max_finite8(xv) : 0);
        }
        if (lane == 0) {
            s_max[0][wave] = mk;
            s_max[1][wave] = mv;
            s_finite[0][wave] = fk;
            s_finite[1][wave] = fv;
        }
    } else if (lane == 0) {
        s_max[0][wave] = s_max[1][wave] = s_finite[0][wave] = s_finite[1][wave] = 0;
    }
    __syncthreads();   // (every thread has also read the held tokens' powers)
    if (block >= 0) {
        uint32_t m = 0, mk = 0, mv = 0;            // infinite values and NaN among them; without
#pragma unroll
        for (int i = 0; i < kWaves; i++) {
            m = max(m, max(s_max[0][i], s_max[1][i]));
            mk = max(mk, s_finite[0][i]);
            mv = max(mv, s_finite[1][i]);
        }
        int kb = power_for(__uint_as_float(mk)), vb = power_for(__uint_as_float(mv));
        const int kh = old & 0xff, vh = old >> 8;
        if (held > 0) {
            kb = min(max(kb, kh), kHighestPower);
            vb = min(max(vb, vh), kHighestPower);
            if (slot < held) {
                if (kb != kh) {
                    const float s = power_of(kh) * power_of(254 - kb);
                    *reinterpret_cast<u32x2_t *>(p.k_pages + code_at) = u32x2_t{scale_codes4(old_k[0], s), scale_codes4(old_k[1], s)};
                }
                if (vb != vh) {
                    const float s = power_of(vh) * power_of(254 - vb);
                    *reinterpret_cast<u32x2_t *>(p.v_pages + code_at) = u32x2_t{scale_codes4(old_v[0], s), scale_codes4(old_v[1], s)};
                }
            }
        }
        if (active) {
            u32x2_t ck, cv;
            float xv[8];
            unpack8(raw_v, xv);
            if (__builtin_expect(m <= __float_as_uint(kLargestCode * 0x1p100f), 1)) {   // all inside their power's range
                ck = codes8(xk, power_of(kb));
                cv = codes8(xv, power_of(vb));
            } else {
                const float ik = power_of(254 - kb), iv = power_of(254 - vb);
                ck = u32x2_t{pack_codes4(xk, ik), pack_codes4(xk + 4, ik)};
                cv = u32x2_t{pack_codes4(xv, iv), pack_codes4(xv + 4, iv)};
            }
            *reinterpret_cast<u32x2_t *>(p.k_pages + code_at) = ck;
            *reinterpret_cast<u32x2_t *>(p.v_pages + code_at) = cv;
        }
        if (threadIdx.x == 0)
            *power = (uint16_t)(kb | vb << 8);
    }
    if (!busy)
        return;
    if (p.q_norm || p.k_norm)
        factors(p.q_norm, q_weights, a, f);
    for (int h0 = 0;;) {
#pragma unroll
        for (int i = 0; i < kQueries; i++) {
            if (h0 + i < p.G) {
                float x[8];
                turned(raw_q[i], p.q_norm, a, f, x);
                if (active)
                    *reinterpret_cast<u32x4_t *>(p.q_out + row * p.q_out_stride + (int64_t)(g * p.G + h0 + i) * D + 8 * c) = pack8(x);
            }
        }
        h0 += kQueries;
        if (h0 >= p.G)
            return;
#pragma unroll
        for (int i = 0; i < kQueries; i++)
            raw_q[i] = load(p.q, p.q_stride, g * p.G + min(h0 + i, p.G - 1));
    }
}

}  // namespace

}  // namespace tsattn

using namespace tsattn;

extern "C" {

int ts_rope_append_kv8(const ts_chunk_shape *s, const ts_rope_config *cfg, const void *q, const void *k, const void *v,
                       void *q_out, void *k_pages, void *v_pages, void *kv_scales, const int32_t *page_table,
                       const int32_t *ctx_lens, const int32_t *q_starts, const float *inv_freq, const void *q_norm,
                       const void *k_norm, void *stream) {
    clear_error();
    int st = check_rope(s, cfg, q, k, v, q_out, k_pages, v_pages, page_table, ctx_lens, q_starts, inv_freq, q_norm,
                        k_norm);
    if (st || s->num_tokens == 0)
        return st;
    if (!kv_scales)
        return fail(TS_ERR_NULL, "kv_scales is NULL");
    if ((uintptr_t)kv_scales & 15)
        return fail(TS_ERR_ARG, "misaligned pointer (16 B needed)");
    if ((st = check_device()))
        return st;
    Rope8Params p;
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.q_out = static_cast<uint16_t *>(q_out);
    p.k_pages = static_cast<uint8_t *>(k_pages);
    p.v_pages = static_cast<uint8_t *>(v_pages);
    p.scales = static_cast<uint8_t *>(kv_scales);
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
    p.G = p.Hq / p.Hkv;
    p.max_pages = s->max_pages_per_seq;
    p.num_tokens = s->num_tokens;
    p.rot = cfg->rot_dim;
    p.eps = cfg->eps;
    const int D = s->head_dim;
    const auto kernel = D == 64 ? cfg->interleaved ? rope_append_kv8_kernel<64, true> : rope_append_kv8_kernel<64, false>
                                : cfg->interleaved ? rope_append_kv8_kernel<128, true> : rope_append_kv8_kernel<128, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(s->num_tokens / kPage + 2 * s->num_seqs), (unsigned)s->num_kv_heads),
                       dim3((unsigned)(kPage * D / 8)), 0, reinterpret_cast<hipStream_t>(stream), p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TS_OK : hip_fail(e, "rotation and 8-bit append launch");
}

}  // extern "C"
