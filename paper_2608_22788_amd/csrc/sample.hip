// sample.hip -- draws each sequence's next token from its row of logits, with
// temperature, top-k, top-p and min-p, from the caller's random numbers.
//
// The rule over real numbers, for a row l, temperature T and uniform u:
//   w_v = exp((l_v - max l) / T);
//   top-k keeps the k largest logits, top-p the largest of those while the
//   mass in front of one is below p times their mass, min-p those with w >=
//   min_p (equal logits rank by index, the lowest first);
//   the token is the smallest v whose running kept mass in index order exceeds
//   u times the kept total Z.
// Where a running mass passes u Z or p Z decides the token, and a vocabulary
// has 10^5 such borders, so masses have to be good to far better than 10^-6 of
// the total: float32 sums would move the draw of about one row in ten.
//
// Masses.  x = l log2(e) / T in float64, n = rint(x), and 2^(x - n) by its
// Taylor polynomial of degree 10 (|x - n| <= 1/2: off by less than 2^-42)
// give a weight's 43-bit significand; relative to a power of two 2^E it is
// that integer shifted right by E - n.  So masses are 64-bit integers in units
// of 2^(E - 42): their sums do not depend on order, thread blocks of different
// E join by a shift, and where the running sum passes a target is found block
// by block, run by run and element by element with the same integers.  A
// weight is off by at most a unit, 2^-42 of the largest.
//
// What bounds it: the row is read once from memory, and a weight costs about
// 20 float64-rate instructions (as many as float32 ones issue here), a little
// less than the read at 4 bytes a logit.  Sequences are few and rows long, so
//   - sample_slices_kernel spreads the rows over the chip in slices, each held
//     in registers: its maximum, then its mass, or, for rows with top-k or
//     top-p, how many logits and how much mass lie in bins of an eighth of a
//     binary order below its maximum (the bins of different slices lie on one
//     grid);
//   - sample_pick_kernel, one workgroup per row, joins the slices and either
//     draws (no filters), or finds the bin where a filter ends, collects the
//     logits above its lower edge into LDS, finds the last kept one there by a
//     radix descent over (logit, index), and draws among the kept ones.
// Only rows whose filter leaves more than fits LDS are read again (from the
// caches).
#include <hip/hip_runtime.h>

#include <cfloat>
#include <climits>

#include "attn_common.h"
#include "ts_attn.h"
#include "ts_internal.h"
#include "wave_scan.h"

// x is rounded before its integer part leaves it; a fused l c - n would not
// belong to the x that n was taken from (fma where it is meant is written out).
#pragma clang fp contract(off)

namespace tsattn {

namespace {

constexpr int kMaxVocabBits = 20;
constexpr int kSliceThreads = 256;
constexpr int kSliceUnit = 16 * kSliceThreads;   // logits of a slice per pass of its registers
constexpr int kLongSlice = 4;                    // passes of the longer slices
constexpr int kBins = 256;
constexpr double kBinsPerOctave = 8.0;
constexpr int kPickThreads = 1024;
constexpr int kPickWaves = kPickThreads / kWave;
constexpr int kRun = 256;                        // logits per mass kept while a filtered row is summed
constexpr int kMaxRuns = (1 << kMaxVocabBits) / kRun;
constexpr int kList = 4096;                      // logits collected in LDS
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;
constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

typedef unsigned long long u64;   // the type of the LDS atomics

struct SampleParams {
    const void *logits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token;
    float *logprob;
    float *s_max;          // [B][slices]
    int32_t *s_arg;        // [B][slices] index of the maximum (greedy rows)
    u64 *s_mass;           // [B][slices] (rows without filters)
    uint32_t *h_count;     // [B][slices][kBins]
    u64 *h_mass;
    int64_t row_stride;
    int V, slices, slice_len;
};

// What a row asks for.
struct RowRule {
    bool greedy, by_k, by_p, by_min;
    double c;       // log2(e) / T
    int k;
    float p, min_p;
};
__device__ __forceinline__ RowRule row_rule(const SampleParams &a, int b) {
    RowRule r;
    const float T = a.temperature ? a.temperature[b] : 1.0f;
    r.greedy = !(T > 0.0f);
    r.c = kLog2e / (double)T;   // 0 for an infinite T: every weight is 1
    r.k = a.top_k ? a.top_k[b] : 0;
    r.by_k = !r.greedy && r.k > 0 && r.k < a.V;
    r.p = a.top_p ? a.top_p[b] : 1.0f;
    r.by_p = !r.greedy && r.p < 1.0f;
    r.min_p = a.min_p ? fminf(a.min_p[b], 1.0f) : 0.0f;
    r.by_min = !r.greedy && r.min_p > 0.0f;
    return r;
}

// ---- logits -----------------------------------------------------------------------
// NaN reads as -inf, +inf as the largest float32, -0 as 0.
__device__ __forceinline__ float clean(float x) { return x > -INFINITY ? fminf(x, FLT_MAX) + 0.0f : -INFINITY; }

// Order-preserving bits of a logit.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// Rank of a logit: a larger one means earlier in descending order with the
// lowest index first.
__device__ __forceinline__ u64 rank_of(float x, int i) {
    return (u64)order_bits(x) << kMaxVocabBits | (u64)((1 << kMaxVocabBits) - 1 - i);
}

// Rows start at any multiple of an element, so vector loads ask for no more
// alignment than that.
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t h8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef uint16_t h4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
__device__ __forceinline__ float one_logit(const T *row, int i) {
    if constexpr (sizeof(T) == 4)
        return clean(row[i]);
    else
        return clean(__uint_as_float((uint32_t)row[i] << 16));
}

// ---- weights ----------------------------------------------------------------------
__device__ __forceinline__ double scaled(float l, double c) { return (double)l * c; }

// The weight of scaled logit x in units of 2^(E - 42) (E >= rint(x)).
__device__ __forceinline__ u64 weight(double x, double E) {
    const double n = rint(x), r = x - n;
    double y = 0x1.e4cf5158b8ec7p+14;            // 2^42 ln(2)^k / k!, k = 10 .. 0
    y = fma(y, r, 0x1.b5253d395e7c1p+18);
    y = fma(y, r, 0x1.62c0223a5c822p+22);
    y = fma(y, r, 0x1.ffcbfc588b0c5p+25);
    y = fma(y, r, 0x1.430912f86c786p+29);
    y = fma(y, r, 0x1.5d87fe78a6730p+32);
    y = fma(y, r, 0x1.3b2ab6fba4e77p+35);
    y = fma(y, r, 0x1.c6b08d704a0bfp+37);
    y = fma(y, r, 0x1.ebfbdff82c58ep+39);
    y = fma(y, r, 0x1.62e42fefa39efp+41);
    // adding 2^52 leaves the integer in the significand
    const double d = fma(y, r, 0x1p52 + 0x1p42);
    const u64 m = (u64)__double_as_longlong(d) & ((1ull << 52) - 1);
    const double s = E - n;
    return s < 64.0 ? m >> (int)s : 0;
}
// (a logit of -inf has no weight; callers test that)

// floor(u z) and ceil(p z) for float32 u, p in [0, 1) and z < 2^63.
__device__ __forceinline__ void fraction_of(float f, u64 z, u64 *floor_out, u64 *ceil_out) {
    const uint32_t bits = __float_as_uint(f), e = bits >> 23;
    const u64 m = e ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
    const int s = e ? 150 - (int)e : 149;        // f = m 2^-s, s >= 24
    const u64 lo = m * z, hi = __umul64hi(m, z); // below 2^87
    u64 q, rest;
    if (s < 64) {
        q = lo >> s | (hi << 1) << (63 - s);
        rest = lo & ((1ull << s) - 1);
    } else {
        const int t = s - 64;
        q = t < 64 ? hi >> t : 0;
        rest = lo | (t < 64 ? hi & ((1ull << t) - 1) : hi);
    }
    *floor_out = q;
    *ceil_out = q + (rest != 0);
}

// ---- block reductions ---------------------------------------------------------------
template <int kWaves>
__device__ __forceinline__ float block_max(float x, float *lds) {
#pragma unroll
    for (int d = 32; d; d >>= 1)
        x = fmaxf(x, __shfl_xor(x, d, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0)
        lds[threadIdx.x / kWave] = x;
    __syncthreads();
    float m = lds[0];
#pragma unroll
    for (int i = 1; i < kWaves; i++)
        m = fmaxf(m, lds[i]);
    __syncthreads();
    return m;
}

// Sum over the block, and this thread's inclusive running sum.
template <int kWaves>
__device__ __forceinline__ u64 block_scan(u64 x, u64 *lds, u64 *total) {
    const u64 incl = wave_incl_scan((uint64_t)x);
    const int wave = threadIdx.x / kWave;
    if ((threadIdx.x & (kWave - 1)) == kWave - 1)
        lds[wave] = incl;
    __syncthreads();
    u64 before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves; i++) {
        const u64 v = lds[i];
        before += i < wave ? v : 0;
        sum += v;
    }
    __syncthreads();
    *total = sum;
    return before + incl;
}

// ---- slices -------------------------------------------------------------------------

template <typename T, int kPasses>
__global__ __launch_bounds__(kSliceThreads) void sample_slices_kernel(SampleParams a) {
    constexpr int kVec = 16 / sizeof(T);                     // logits per load
    constexpr int kLoads = 16 * kPasses / kVec;
    __shared__ float red[kSliceThreads / kWave];
    __shared__ u64 mass_of[kBins], wave_mass[kSliceThreads / kWave];
    __shared__ uint32_t count_of[kBins];
    __shared__ int arg;
    const int b = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const int tid = threadIdx.x;
    const RowRule rule = row_rule(a, b);
    const int first = slice * a.slice_len, n = min(a.V - first, a.slice_len);
    const T *src = static_cast<const T *>(a.logits) + (int64_t)b * a.row_stride + first;

    float l[kLoads][kVec];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = (i * kSliceThreads + tid) * kVec;
        if (at + kVec <= n) {
            if constexpr (sizeof(T) == 4) {
                const f4_any v = *reinterpret_cast<const f4_any *>(src + at);
#pragma unroll
                for (int e = 0; e < kVec; e++)
                    l[i][e] = clean(v[e]);
            } else {
                const h8_any v = *reinterpret_cast<const h8_any *>(src + at);
#pragma unroll
                for (int e = 0; e < kVec; e++)
                    l[i][e] = clean(__uint_as_float((uint32_t)v[e] << 16));
            }
        } else {
#pragma unroll
            for (int e = 0; e < kVec; e++)
                l[i][e] = at + e < n ? one_logit(src, at + e) : -INFINITY;
        }
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLoads; i++)
#pragma unroll
        for (int e = 0; e < kVec; e++)
            m = fmaxf(m, l[i][e]);
    m = block_max<kSliceThreads / kWave>(m, red);
    const size_t at_slice = (size_t)b * a.slices + slice;
    if (tid == 0)
        a.s_max[at_slice] = m;
    if (rule.greedy) {
        if (tid == 0)
            arg = INT_MAX;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads; i++)
#pragma unroll
            for (int e = 0; e < kVec; e++)
                if (l[i][e] == m)
                    atomicMin(&arg, first + (i * kSliceThreads + tid) * kVec + e);
        __syncthreads();
        if (tid == 0)
            a.s_arg[at_slice] = arg;
        return;
    }
    const double top = scaled(m, rule.c), E = rint(top);
    if (!rule.by_k && !rule.by_p) {
        if (rule.by_min)
            return;   // the maximum is all that the pick needs
        u64 sum = 0;
        if (m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kLoads; i++)
#pragma unroll
                for (int e = 0; e < kVec; e++)
                    sum += l[i][e] > -INFINITY ? weight(scaled(l[i][e], rule.c), E) : 0;
        }
        u64 total;
        block_scan<kSliceThreads / kWave>(sum, wave_mass, &total);
        if (tid == 0)
            a.s_mass[at_slice] = total;
        return;
    }
    static_assert(kBins == kSliceThreads, "one bin per thread");
    count_of[tid] = 0;
    mass_of[tid] = 0;
    __syncthreads();
    const double top_bin = floor(top * kBinsPerOctave);
#pragma unroll
    for (int i = 0; i < kLoads; i++)
#pragma unroll
        for (int e = 0; e < kVec; e++)
            if (l[i][e] > -INFINITY) {
                const double x = scaled(l[i][e], rule.c);
                const int bin = (int)fmin(top_bin - floor(x * kBinsPerOctave), (double)(kBins - 1));
                atomicAdd(&count_of[bin], 1u);
                if (rule.by_p)
                    atomicAdd(&mass_of[bin], weight(x, E));
            }
    __syncthreads();
    a.h_count[at_slice * kBins + tid] = count_of[tid];
    if (rule.by_p)
        a.h_mass[at_slice * kBins + tid] = mass_of[tid];
}

// ---- pick ---------------------------------------------------------------------------

struct PickLds {
    u64 list[kList];        // ranks of the collected logits
    u64 digit[kDigits];
    u64 run[kMaxRuns];      // kept mass of each run of logits
    u64 waves[kPickWaves];
    u64 bin_mass[kBins];
    uint32_t bin_count[kBins];
    float red[kPickWaves];
    u64 found64, found_base;
    int found, last, n;
};

// First index i of v[0 .. n) whose running sum reaches `target` (n if none), in
// every thread; *base is the sum in front of it.  n <= kPer * threads.
template <int kPer, typename Get>
__device__ __forceinline__ int first_reaching(PickLds &s, int n, u64 target, u64 *base, u64 *total, Get get) {
    const int tid = threadIdx.x;
    u64 v[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int at = kPer * tid + i;
        v[i] = at < n ? get(at) : 0;
        sum += v[i];
    }
    if (tid == 0)
        s.found = n;
    const u64 incl = block_scan<kPickWaves>(sum, s.waves, total);
    u64 acc = incl - sum;
    if (acc < target && incl >= target) {
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            if (acc < target && acc + v[i] >= target) {
                s.found = kPer * tid + i;
                s.found_base = acc;
            }
            acc += v[i];
        }
    }
    __syncthreads();
    const int f = s.found;
    *base = f < n ? s.found_base : 0;
    __syncthreads();
    return f;
}

// Lowest logit of bin `bin` or a bin above it: the smallest float32 l with
// floor(x(l) bins) >= top - bin.  The quotient is within a step of it.
__device__ __forceinline__ float bin_edge(double top_bin, int bin, double c) {
    if (bin >= kBins - 1)
        return -FLT_MAX;
    const double want = top_bin - bin;
    const double at = want / (kBinsPerOctave * c);
    const float guess = at > -FLT_MAX ? at < FLT_MAX ? (float)at : FLT_MAX : -FLT_MAX;
    const auto in = [&](float l) { return floor(scaled(l, c) * kBinsPerOctave) >= want; };
    uint32_t k = order_bits(guess + 0.0f);
    const uint32_t low = order_bits(-FLT_MAX), high = order_bits(FLT_MAX);
    for (int i = 0; i < 4 && k > low && in(from_order_bits(k)); i++)
        k--;
    for (int i = 0; i < 8 && k < high && !in(from_order_bits(k)); i++)
        k++;
    return from_order_bits(k);
}

// Calls f(l, i) for every logit of the row (whole workgroup; a wavefront takes
// runs of kRun consecutive ones, a lane four of them).
template <typename T, typename F>
__device__ __forceinline__ void for_row(const T *row, int V, F f) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const int runs = (V + kRun - 1) / kRun;
    constexpr int kAhead = 4;
    for (int r0 = wave; r0 < runs; r0 += kAhead * kPickWaves) {
        float l[kAhead][4];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int at = (r0 + i * kPickWaves) * kRun + 4 * lane;
            if (at + 4 <= V) {
                if constexpr (sizeof(T) == 4) {
                    const f4_any v = *reinterpret_cast<const f4_any *>(row + at);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        l[i][e] = clean(v[e]);
                } else {
                    const h4_any v = *reinterpret_cast<const h4_any *>(row + at);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        l[i][e] = clean(__uint_as_float((uint32_t)v[e] << 16));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    l[i][e] = at + e < V ? one_logit(row, at + e) : -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++)
            if (r0 + i * kPickWaves < runs)
                f(r0 + i * kPickWaves, l[i], (r0 + i * kPickWaves) * kRun + 4 * lane);
    }
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleParams a) {
    extern __shared__ u64 pick_lds[];
    PickLds &s = *reinterpret_cast<PickLds *>(pick_lds);
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & (kWave - 1);
    const RowRule rule = row_rule(a, b);
    const size_t slice0 = (size_t)b * a.slices;
    const T *row = static_cast<const T *>(a.logits) + (int64_t)b * a.row_stride;

    float m = -INFINITY;
    for (int i = tid; i < a.slices; i += kPickThreads)
        m = fmaxf(m, a.s_max[slice0 + i]);
    m = block_max<kPickWaves>(m, s.red);
    if (!(m > -INFINITY)) {   // nothing to draw from
        if (tid == 0) {
            a.token[b] = -1;
            if (a.logprob)
                a.logprob[b] = -INFINITY;
        }
        return;
    }
    if (rule.greedy) {
        if (tid == 0)
            s.found = INT_MAX;
        __syncthreads();
        for (int i = tid; i < a.slices; i += kPickThreads)
            if (a.s_max[slice0 + i] == m)
                atomicMin(&s.found, a.s_arg[slice0 + i]);
        __syncthreads();
        if (tid == 0) {
            a.token[b] = s.found;
            if (a.logprob)
                a.logprob[b] = 0.0f;
        }
        return;
    }

    const double c = rule.c, top = scaled(m, c), E = rint(top);
    const float u = a.u[b] > 0.0f ? fminf(a.u[b], 0x1.fffffep-1f) : 0.0f;
    u64 Z = 0, base = 0, unused, target;
    int run, run_len;
    double run_E = E;         // the unit of the weights inside the chosen run
    u64 cut = 0;              // lowest rank that is kept
    float low = -FLT_MAX;     // no logit below it is kept
    const double min_x = rule.by_min ? log2((double)rule.min_p) : 0.0;
    const auto passes_min = [&](float l) { return !rule.by_min || ((double)l - (double)m) * c >= min_x; };

    if (!rule.by_k && !rule.by_p && !rule.by_min) {
        // the slices' masses in the row's unit
        for (int i = tid; i < a.slices; i += kPickThreads) {
            const float sm = a.s_max[slice0 + i];
            const double d = sm > -INFINITY ? E - rint(scaled(sm, c)) : 64.0;
            s.run[i] = d < 64.0 ? a.s_mass[slice0 + i] >> (int)d : 0;
        }
        __syncthreads();
        run_len = a.slice_len;
        run = first_reaching<1>(s, a.slices, 1, &base, &Z, [&](int i) { return s.run[i]; });
        fraction_of(u, Z, &target, &unused);
        run = first_reaching<1>(s, a.slices, target + 1, &base, &Z, [&](int i) { return s.run[i]; });
        run = min(run, a.slices - 1);
        run_E = rint(scaled(a.s_max[slice0 + run], c));
        target = (target - base) << (int)(E - run_E);
    } else {
        bool listed = false;
        if (rule.by_k || rule.by_p) {
            // the slices' bins on the row's grid
            for (int i = tid; i < kBins; i += kPickThreads) {
                s.bin_count[i] = 0;
                s.bin_mass[i] = 0;
            }
            __syncthreads();
            const double top_bin = floor(top * kBinsPerOctave);
            for (int i = tid; i < a.slices * kBins; i += kPickThreads) {
                const float sm = a.s_max[slice0 + i / kBins];
                const uint32_t n = a.h_count[slice0 * kBins + i];
                if (n == 0)
                    continue;
                const double stop = scaled(sm, c);
                const double off = top_bin - floor(stop * kBinsPerOctave), d = E - rint(stop);
                const int bin = (int)fmin(off + i % kBins, (double)(kBins - 1));
                atomicAdd(&s.bin_count[bin], n);
                if (rule.by_p && d < 64.0)
                    atomicAdd(&s.bin_mass[bin], a.h_mass[slice0 * kBins + i] >> (int)d);
            }
            __syncthreads();

            // the bin in which a running sum reaches a target: the filter's last one
            u64 above = 0, all = 0;
            u64 want = rule.k;
            bool by_count = rule.by_k;
            int bin = kBins;
            if (rule.by_k)
                bin = first_reaching<1>(s, kBins, want, &above, &all, [&](int i) { return (u64)s.bin_count[i]; });
            if (bin == kBins) {   // top-k off, or no fewer than the row has
                by_count = false;
                if (rule.by_p) {
                    first_reaching<1>(s, kBins, 1, &above, &all, [&](int i) { return s.bin_mass[i]; });
                    fraction_of(fmaxf(rule.p, 0.0f), all, &unused, &want);
                    want = want > 0 ? want : 1;
                    bin = first_reaching<1>(s, kBins, want, &above, &all, [&](int i) { return s.bin_mass[i]; });
                    bin = min(bin, kBins - 1);
                }
            }
            const bool then_p = by_count && rule.by_p;
            if (bin < kBins) {
                u64 n;
                first_reaching<1>(s, bin + 1, ~0ull, &base, &n, [&](int i) { return (u64)s.bin_count[i]; });
                listed = n <= kList;
                low = bin_edge(top_bin, bin, c);
                // in front of what a descent looks at: everything above the
                // bin, unless the list (or a top-p after a top-k) holds that too
                const bool whole = listed || then_p;
                const float high = whole || bin == 0 ? INFINITY : bin_edge(top_bin, bin - 1, c);
                if (!whole)
                    want -= above;
                if (tid == 0)
                    s.n = 0;
                __syncthreads();
                if (listed) {
                    for_row(row, a.V, [&](int, const float(&l)[4], int at) {
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (l[e] >= low) {
                                const int i = atomicAdd(&s.n, 1);
                                if (i < kList)   // (the bins counted no more)
                                    s.list[i] = rank_of(l[e], at + e);
                            }
                    });
                    __syncthreads();
                }
                const int n_list = min(s.n, kList);
                // Runs f(rank, logit) over the list, or over the row's logits in [low, high).
                const auto for_candidates = [&](auto f) {
                    if (listed) {
                        for (int i = tid; i < n_list; i += kPickThreads)
                            f(s.list[i], from_order_bits((uint32_t)(s.list[i] >> kMaxVocabBits)));
                    } else {
                        for_row(row, a.V, [&](int, const float(&l)[4], int at) {
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                if (l[e] >= low && l[e] < high)
                                    f(rank_of(l[e], at + e), l[e]);
                        });
                    }
                };
                // The rank at which the running sum (of counts, or of weights) reaches `want`.
                const auto descend = [&](bool counts, u64 want) {
                    u64 prefix = 0;
                    for (int shift = 32 + kMaxVocabBits; shift > 0;) {
                        const int next = max(shift - kDigitBits, 0), digits = 1 << (shift - next);
                        for (int i = tid; i < kDigits; i += kPickThreads)
                            s.digit[i] = 0;
                        __syncthreads();
                        for_candidates([&](u64 rank, float l) {
                            if (shift == 32 + kMaxVocabBits || rank >> shift == prefix)
                                atomicAdd(&s.digit[digits - 1 - ((rank >> next) & (digits - 1))],
                                          counts ? 1ull : weight(scaled(l, c), E));
                        });
                        __syncthreads();
                        u64 in_front, sum;
                        int d = first_reaching<kDigits / kPickThreads>(s, digits, want, &in_front, &sum,
                                                                       [&](int i) { return s.digit[i]; });
                        if (d == digits) {   // short by rounding of the bins' masses: the last one
                            want = sum;
                            d = first_reaching<kDigits / kPickThreads>(s, digits, want, &in_front, &sum,
                                                                       [&](int i) { return s.digit[i]; });
                            d = min(d, digits - 1);
                        }
                        want -= in_front;
                        prefix = prefix << (shift - next) | (u64)(digits - 1 - d);
                        shift = next;
                    }
                    return prefix;
                };
                cut = descend(by_count, want);
                if (then_p) {
                    u64 kept = 0;
                    for_candidates([&](u64 rank, float l) { kept += rank >= cut ? weight(scaled(l, c), E) : 0; });
                    block_scan<kPickWaves>(kept, s.waves, &all);
                    fraction_of(fmaxf(rule.p, 0.0f), all, &unused, &want);
                    const u64 cut_p = descend(false, want > 0 ? want : 1);
                    cut = cut_p > cut ? cut_p : cut;
                }
            }
        }
        // the kept mass of every run
        const int runs = (a.V + kRun - 1) / kRun;
        run_len = kRun;
        if (listed) {
            for (int i = tid; i < runs; i += kPickThreads)
                s.run[i] = 0;
            __syncthreads();
            const int n_list = min(s.n, kList);
            for (int i = tid; i < n_list; i += kPickThreads) {
                const u64 rank = s.list[i];
                const float l = from_order_bits((uint32_t)(rank >> kMaxVocabBits));
                if (rank >= cut && passes_min(l))
                    atomicAdd(&s.run[((1 << kMaxVocabBits) - 1 - (int)(rank & ((1 << kMaxVocabBits) - 1))) / kRun],
                              weight(scaled(l, c), E));
            }
        } else {
            if (cut)
                low = fmaxf(low, from_order_bits((uint32_t)(cut >> kMaxVocabBits)));
            if (rule.by_min) {   // one float32 below where min-p ends, whichever way that rounds
                const double at = (double)m + min_x / c;
                if (at > -(double)FLT_MAX)
                    low = fmaxf(low, from_order_bits(order_bits((float)at + 0.0f) - 1));
            }
            for_row(row, a.V, [&](int r, const float(&l)[4], int at) {
                u64 sum = 0;
                if (__any(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= low)) {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (l[e] >= low && rank_of(l[e], at + e) >= cut && passes_min(l[e]))
                            sum += weight(scaled(l[e], c), E);
                    sum = wave_incl_scan((uint64_t)sum);
                }
                if (lane == kWave - 1)
                    s.run[r] = sum;
            });
        }
        __syncthreads();
        run = first_reaching<kMaxRuns / kPickThreads>(s, runs, 1, &base, &Z, [&](int i) { return s.run[i]; });
        fraction_of(u, Z, &target, &unused);
        run = first_reaching<kMaxRuns / kPickThreads>(s, runs, target + 1, &base, &Z, [&](int i) { return s.run[i]; });
        run = min(run, runs - 1);
        target -= base;
    }

    // the token inside the run: the first whose running weight exceeds the target
    const int per = (run_len + kPickThreads - 1) / kPickThreads;
    const int at = run * run_len + tid * per, end = min(min(at + per, (run + 1) * run_len), a.V);
    const auto kept_weight = [&](int i) -> u64 {
        const float l = one_logit(row, i);
        return l > -INFINITY && rank_of(l, i) >= cut && passes_min(l) ? weight(scaled(l, c), run_E) : 0;
    };
    u64 sum = 0;
    int last = -1;
    for (int i = at; i < end; i++) {
        const u64 w = kept_weight(i);
        sum += w;
        last = w ? i : last;
    }
    if (tid == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    u64 total;
    const u64 incl = block_scan<kPickWaves>(sum, s.waves, &total);
    if (last >= 0)
        atomicMax(&s.last, last);   // what rounding of a slice's shift may leave as the answer
    u64 acc = incl - sum;
    if (acc <= target && incl > target) {
        int i = at;
        for (; i < end; i++) {
            acc += kept_weight(i);
            if (acc > target)
                break;
        }
        s.found = i;
    }
    __syncthreads();
    if (tid == 0) {
        const int token = s.found < a.V ? s.found : s.last;
        a.token[b] = token;
        if (a.logprob)
            a.logprob[b] = token < 0 ? -INFINITY
                                     : (float)((scaled(one_logit(row, token), c) - E) * kLn2 - log((double)Z * 0x1p-42));
    }
}

struct SamplePlan {
    int slices, slice_len;
    size_t arg_off, mass_off, count_off, hmass_off, bytes;
};

// Short slices spread few rows over the chip; from 2,048 workgroups on longer
// ones keep the bins (3 KiB a slice) small beside the logits.
int make_sample_plan(int32_t B, int32_t V, SamplePlan *pl) {
    if (B < 1 || B > 65536)
        return fail(TS_ERR_ARG, "num_seqs %d outside [1, 65536]", B);
    if (V < 1 || V > (1 << kMaxVocabBits))
        return fail(TS_ERR_ARG, "vocab %d outside [1, 2^20]", V);
    const int64_t shorter = ((int64_t)V + kSliceUnit - 1) / kSliceUnit;
    pl->slice_len = B * shorter <= 2048 ? kSliceUnit : kLongSlice * kSliceUnit;
    pl->slices = (V + pl->slice_len - 1) / pl->slice_len;
    const size_t n = (size_t)B * pl->slices;
    const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    pl->arg_off = up(n * sizeof(float));
    pl->mass_off = pl->arg_off + up(n * sizeof(int32_t));
    pl->count_off = pl->mass_off + up(n * sizeof(u64));
    pl->hmass_off = pl->count_off + up(n * kBins * sizeof(uint32_t));
    pl->bytes = pl->hmass_off + up(n * kBins * sizeof(u64));
    return TS_OK;
}

template <typename T>
hipError_t launch_sample(const SampleParams &a, int B, hipStream_t hs) {
    const auto slices = a.slice_len == kSliceUnit ? sample_slices_kernel<T, 1> : sample_slices_kernel<T, kLongSlice>;
    hipLaunchKernelGGL(slices, dim3((unsigned)B * (unsigned)a.slices), dim3(kSliceThreads), 0, hs, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(sample_pick_kernel<T>, dim3((unsigned)B), dim3(kPickThreads), sizeof(PickLds), hs, a);
    return hipGetLastError();
}

}  // namespace

}  // namespace tsattn

using namespace tsattn;

extern "C" {

size_t ts_sample_workspace_size(int32_t num_seqs, int32_t vocab) {
    clear_error();
    SamplePlan pl;
    return make_sample_plan(num_seqs, vocab, &pl) == TS_OK ? pl.bytes : 0;
}

int ts_sample(int32_t num_seqs, int32_t vocab, int32_t logits_type, const void *logits, int64_t row_stride,
              const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
              int32_t *token, float *logprob, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    SamplePlan pl;
    int st = make_sample_plan(num_seqs, vocab, &pl);
    if (st)
        return st;
    if (!logits || !u || !token || !workspace)
        return fail(TS_ERR_NULL, "a pointer is NULL");
    if (logits_type != TS_LOGITS_F32 && logits_type != TS_LOGITS_BF16)
        return fail(TS_ERR_ARG, "logits_type %d unknown", logits_type);
    if (row_stride < vocab || row_stride > (1LL << 32))
        return fail(TS_ERR_ARG, "row_stride %lld outside [vocab, 2^32]", (long long)row_stride);
    if (workspace_bytes < pl.bytes)
        return fail(TS_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, pl.bytes);
    if (((uintptr_t)logits & (logits_type == TS_LOGITS_F32 ? 3 : 1)) || ((uintptr_t)workspace & 255))
        return fail(TS_ERR_ARG, "misaligned pointer (logits an element, workspace 256 B)");
    if ((st = check_device()))
        return st;
    char *ws = static_cast<char *>(workspace);
    SampleParams a;
    a.logits = logits;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.u = u;
    a.token = token;
    a.logprob = logprob;
    a.s_max = reinterpret_cast<float *>(ws);
    a.s_arg = reinterpret_cast<int32_t *>(ws + pl.arg_off);
    a.s_mass = reinterpret_cast<u64 *>(ws + pl.mass_off);
    a.h_count = reinterpret_cast<uint32_t *>(ws + pl.count_off);
    a.h_mass = reinterpret_cast<u64 *>(ws + pl.hmass_off);
    a.row_stride = row_stride;
    a.V = vocab;
    a.slices = pl.slices;
    a.slice_len = pl.slice_len;
    hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    const hipError_t e = logits_type == TS_LOGITS_F32 ? launch_sample<float>(a, num_seqs, hs)
                                                      : launch_sample<uint16_t>(a, num_seqs, hs);
    return e == hipSuccess ? TS_OK : hip_fail(e, "sampling launch");
}

}  // extern "C"
