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
// Taylor polynomial of degree 10 give a weight's 43-bit significand; relative to
// a power of two 2^E it is that integer shifted right by E - n.  So masses are
// 64-bit integers in units of 2^(E - 42), at most 2^-41.5 of the largest weight:
// their sums do not depend on order, thread blocks of different E join by a
// shift, and where the running sum passes a target is found block by block, run
// by run and element by element with the same integers.  The significand is off
// by at most 1.48 (the series' end 0.98 at |x - n| = 1/2, its rounding 0.5), so a
// weight by 1.5 units, the shift included.  x is rounded at its own size, not at
// its distance from the maximum: by 2^-53 |l / T| of the weight, which passes a
// unit for the largest ones where |l / T| passes about 2,000.
//
// What bounds it: the row is read once from memory, and a weight costs 22
// float64-rate instructions (as many as float32 ones issue here), about as
// long as reading 4 bytes takes.  Sequences are few and rows long, so the work
// on whole rows is spread over the chip in slices held in registers:
//   - sample_slices_kernel: a slice's maximum, then its mass, or, for rows with
//     top-k or top-p, how many logits and how much mass lie in bins of an
//     eighth of a binary order below its maximum (the bins of different slices
//     lie on one grid);
//   - sample_plan_kernel, one workgroup per row, joins the slices and draws
//     where there is no filter; else it finds the bin where the filter ends;
// and with filters
//   - sample_gather_kernel appends the logits from that bin on to the row's
//     list, or, where they are many, the bin's alone (what lies above it is then
//     summed from the bins, or here where they hold no masses);
//   - sample_filter_kernel, one workgroup per row, finds the last kept logit in
//     the list (pair by pair if few, else by a radix descent over (logit,
//     index)) and draws.
// Measured, 151,936 logits a row: 8 float32 rows with temperature alone 12.4
// us; 200 bf16 rows, each with its own filters, 94 us (kernels 42, 10, 20 and 25
// us; with one workgroup reading each filtered row again instead of the last
// two kernels' slices it was 245 us).  200 rows, every one with top-k 50: 59-64
// us, top-p 0.9: 95-107, min-p 0.05: 42-55, none: 41, of which the weights'
// arithmetic is the largest part (slices 34; reading them alone 12.6).  48
// float32 rows of 50,257 with top-p: 41 us, the chain of four launches.  Only a
// row of which more than kList logits lie in one bin is still read by one
// workgroup: 8 float32 rows with top-p take 44 us just short of that, 265 past it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

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
constexpr int kLongSlice = 2;                    // passes of the longer slices
constexpr int kBins = 256;
constexpr double kBinsPerOctave = 8.0;
constexpr int kMaxSlices = (1 << kMaxVocabBits) / kSliceUnit;
constexpr int kPlanThreads = 1024, kFilterThreads = 1024;
constexpr int kRun = 256;                        // logits that a wavefront reads at once of a whole row
constexpr int kList = 8192;                      // candidates of a row
constexpr int kFew = 256;                        // of them, compared pair by pair
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;

constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

typedef unsigned long long u64;   // the type of the LDS atomics

// What the filters leave to be found out about a row (see sample_plan_kernel).
enum { kDrawn, kListed, kScanned };   // done; candidates in the list; too many of them
struct RowPlan {
    int state;
    int n;                  // candidates appended to the list
    float m;                // largest logit
    float lo, hi;
    bool by_count, then_p;  // a top-k ends among the candidates; then a top-p of what it keeps
    bool summed;            // s_mass holds what is kept of each slice above the candidates
    u64 want;               // the running count or mass at which the filter ends (0: none does)
};

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
    RowPlan *plan;         // [B]
    u64 *list;             // [B][list_len]
    int64_t row_stride;
    int V, slices, slice_len, list_len;
};

// What a row asks for.
struct RowRule {
    bool greedy, by_k, by_p, by_min;
    double c;       // log2(e) / T
    int k;
    float p;
    double min_x;   // log2(min_p)
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
    const float min_p = a.min_p ? a.min_p[b] : 0.0f;
    r.by_min = !r.greedy && min_p > 0.0f;   // (not for NaN)
    r.min_x = r.by_min ? log2((double)fminf(min_p, 1.0f)) : 0.0;
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

// A constant in scalar registers, where the compiler would otherwise move it
// into the accumulator of every multiply-add (two moves each).
__device__ __forceinline__ double scalar(double k) {
    asm("" : "+s"(k));
    return k;
}

// The weight of scaled logit x in units of 2^(E - 42) (E >= rint(x)); 0 for the
// -inf or NaN that x is for a logit of -inf.
__device__ __forceinline__ u64 weight(double x, double E) {
    constexpr double k[11] = {0x1p52 + 0x1p42, 0x1.62e42fefa39efp+41, 0x1.ebfbdff82c58ep+39, 0x1.c6b08d704a0bfp+37, 0x1.3b2ab6fba4e77p+35, 0x1.5d87fe78a6730p+32,
                              0x1.430912f86c786p+29, 0x1.ffcbfc588b0c5p+25, 0x1.62c0223a5c822p+22, 0x1.b5253d395e7c1p+18, 0x1.e4cf5158b8ec7p+14};   // 2^42 ln(2)^i / i!
    const double n = rint(x), r = x - n;
    double y = scalar(k[10]);
#pragma unroll
    for (int i = 9; i >= 0; i--)
        y = fma(y, r, scalar(k[i]));
    // adding 2^52 has left the integer in the significand
    const u64 m = (u64)__double_as_longlong(y) & ((1ull << 52) - 1);
    const double s = E - n;
    return s < 64.0 ? m >> (int)s : 0;
}

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

// The n logits of a slice, -inf past them: thread t holds kVec from index
// (i * kSliceThreads + t) * kVec.
template <typename T, int kPasses>
__device__ __forceinline__ void load_slice(const T *src, int n, float (&l)[16 * kPasses * sizeof(T) / 16][16 / sizeof(T)]) {
    constexpr int kVec = 16 / sizeof(T), kLoads = 16 * kPasses / kVec;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = (i * kSliceThreads + (int)threadIdx.x) * kVec;
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
    load_slice<T, kPasses>(src, n, l);
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
#pragma unroll
        for (int i = 0; i < kLoads; i++)
#pragma unroll
            for (int e = 0; e < kVec; e++)
                sum += weight(scaled(l[i][e], rule.c), E);
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
    uint32_t far = 0;   // what lies in the last bin, most logits of a confident row, is summed in registers
    u64 far_mass = 0;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        // (no branch per logit, so that the weights' chains run beside each other)
        int bin[kVec];
        u64 w[kVec];
#pragma unroll
        for (int e = 0; e < kVec; e++)
            bin[e] = (int)fmin(top_bin - floor(scaled(l[i][e], rule.c) * kBinsPerOctave), kBins - 1.0);
        if (rule.by_p) {
#pragma unroll
            for (int e = 0; e < kVec; e++) {
                w[e] = weight(scaled(l[i][e], rule.c), E);
                far_mass += bin[e] == kBins - 1 ? w[e] : 0;
            }
#pragma unroll
            for (int e = 0; e < kVec; e++)
                if (bin[e] < kBins - 1)
                    atomicAdd(&mass_of[bin[e]], w[e]);
        }
        if (rule.by_k) {
#pragma unroll
            for (int e = 0; e < kVec; e++) {
                far += bin[e] == kBins - 1 && l[i][e] > -INFINITY;
                if (bin[e] < kBins - 1)
                    atomicAdd(&count_of[bin[e]], 1u);
            }
        }
    }
    if (far)
        atomicAdd(&count_of[kBins - 1], far);
    if (far_mass)
        atomicAdd(&mass_of[kBins - 1], far_mass);
    __syncthreads();
    if (rule.by_k)
        a.h_count[at_slice * kBins + tid] = count_of[tid];
    if (rule.by_p)
        a.h_mass[at_slice * kBins + tid] = mass_of[tid];
}

// ---- pick ---------------------------------------------------------------------------

// What every pick workgroup needs in LDS, and what the filters' ones need.
struct DrawLds {
    u64 waves[kFilterThreads / kWave];
    float red[kFilterThreads / kWave];
    u64 found_base;
    int found, last;
};
struct PlanLds : DrawLds {
    u64 bin_mass[kBins];
    uint32_t bin_count[kBins];
    int bins_off[kMaxSlices], shift[kMaxSlices];
    u64 n_low, n_bin;
};
struct FilterLds : DrawLds {
    u64 list[kList];        // ranks of the candidates
    u64 weight[kList];
    u64 digit[kDigits];     // sums by digit
    u64 slice[kMaxSlices];  // kept mass of each slice
    u64 few[kFew], few_weight[kFew];   // candidates that share the digits found so far
    u64 differ, cut;
    int n;
};

// First index i of the n values get(i) whose running sum reaches a target that
// may depend on their total (n if none), in every thread; *base is the sum in
// front of it.  n <= kPer * threads.
template <int kThreads, int kPer, typename Get, typename Target>
__device__ __forceinline__ int first_reaching(DrawLds &s, int n, u64 *base, u64 *total, u64 *target, Get get, Target target_of) {
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
    const u64 incl = block_scan<kThreads / kWave>(sum, s.waves, total);
    const u64 want = target_of(*total);
    u64 acc = incl - sum;
    if (acc < want && incl >= want) {
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            if (acc < want && acc + v[i] >= want) {
                s.found = kPer * tid + i;
                s.found_base = acc;
            }
            acc += v[i];
        }
    }
    __syncthreads();
    const int f = s.found;
    *base = f < n ? s.found_base : 0;
    *target = want;
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

// Calls f(run, l, i) for the logits of the row, l[0 .. 3] from index i (whole
// workgroup; a wavefront takes runs of kRun consecutive ones, a lane four).
template <typename T, typename F>
__device__ __forceinline__ void for_row(const T *row, int V, F f) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const int runs = (V + kRun - 1) / kRun;
    constexpr int kAhead = 4, kWaves = kFilterThreads / kWave;
    for (int r0 = wave; r0 < runs; r0 += kAhead * kWaves) {
        float l[kAhead][4];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int at = (r0 + i * kWaves) * kRun + 4 * lane;
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
            if (r0 + i * kWaves < runs)
                f(r0 + i * kWaves, l[i], (r0 + i * kWaves) * kRun + 4 * lane);
    }
}

// Sum over kEach neighbouring lanes, in each of them.
constexpr int kEach = kFilterThreads / kFew;
__device__ __forceinline__ u64 sum_each(u64 x) {
#pragma unroll
    for (int d = 1; d < kEach; d *= 2)
        x += __shfl_xor(x, d, kWave);
    return x;
}

__device__ __forceinline__ float clamp_u(float u) { return u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f; }

// The running mass that the drawn token is the first to reach.
__device__ __forceinline__ u64 draw_target(float u, u64 total) {
    u64 lo, up;
    fraction_of(u, total, &lo, &up);
    return lo + 1;
}
// The running mass that the last token of a top-p is the first to reach.
__device__ __forceinline__ u64 p_target(const RowRule &rule, u64 total) {
    u64 lo, up;
    fraction_of(fmaxf(rule.p, 0.0f), total, &lo, &up);
    return up > 0 ? up : 1;
}

// min-p is w >= min_p on the logits' exact distance from the largest, m.
__device__ __forceinline__ bool passes_min(const RowRule &rule, float l, float m) {
    return !rule.by_min || ((double)l - (double)m) * rule.c >= rule.min_x;
}
// A logit below which nothing passes: one float32 below where min-p ends,
// whichever way that rounds.
__device__ __forceinline__ float min_p_edge(const RowRule &rule, float m) {
    const double at = (double)m + rule.min_x / rule.c;
    return at > -(double)FLT_MAX ? from_order_bits(order_bits((float)at + 0.0f) - 1) : -FLT_MAX;
}

// A row whose maximum is known.
struct Row {
    int b;
    float m;          // largest logit
    double c, E;      // log2(e) / T; weights are in units of 2^(E - 42)
    float u;
};

__device__ __forceinline__ void write_token(const SampleParams &a, const Row &r, int token, float l, u64 Z) {
    a.token[r.b] = token;
    if (a.logprob)
        a.logprob[r.b] = token < 0 ? -INFINITY : (float)((scaled(l, r.c) - r.E) * kLn2 - log((double)Z * 0x1p-42));
}

// The token inside a run of `len` logits from `first`: the first whose running
// weight exceeds `target`; weights (get) are in the run's own unit.
template <int kThreads, typename T, typename Get>
__device__ __forceinline__ void draw_inside(const SampleParams &a, const Row &r, const T *row, DrawLds &s, int first, int len,
                                            u64 target, u64 Z, Get get) {
    const int tid = threadIdx.x;
    const int per = (len + kThreads - 1) / kThreads;
    const int at = first + tid * per, end = min(min(at + per, first + len), a.V);
    u64 sum = 0;
    int last = -1;
    for (int i = at; i < end; i++) {
        const u64 w = get(i);
        sum += w;
        last = w ? i : last;
    }
    if (tid == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    u64 total;
    const u64 incl = block_scan<kThreads / kWave>(sum, s.waves, &total);
    if (total <= target && last >= 0)
        atomicMax(&s.last, last);   // a run's shifted mass was a unit more than its weights
    u64 acc = incl - sum;
    if (acc <= target && incl > target) {
        int i = at;
        for (; i < end; i++) {
            acc += get(i);
            if (acc > target)
                break;
        }
        s.found = i;
    }
    __syncthreads();
    if (tid == 0) {
        const int token = s.found < a.V ? s.found : s.last;
        write_token(a, r, token, token < 0 ? 0.0f : one_logit(row, token), Z);
    }
}

// Rows that need no filter: the largest logit, or the draw by the slices'
// masses.  Returns whether the row was such a one.
template <int kThreads, typename T>
__device__ __forceinline__ bool draw_unfiltered(const SampleParams &a, const RowRule &rule, Row &r, const T *row, DrawLds &s) {
    const int tid = threadIdx.x;
    const size_t slice0 = (size_t)r.b * a.slices;
    static_assert(kMaxSlices <= kPlanThreads, "one slice per thread");
    const float sm = tid < a.slices ? a.s_max[slice0 + tid] : -INFINITY;
    const u64 mass = tid < a.slices ? a.s_mass[slice0 + tid] : 0;   // (of a greedy or filtered row: not used)
    r.u = clamp_u(a.u[r.b]);
    r.m = block_max<kThreads / kWave>(sm, s.red);
    r.c = rule.c;
    if (!(r.m > -INFINITY)) {   // nothing to draw from
        if (tid == 0)
            write_token(a, r, -1, 0.0f, 0);
        return true;
    }
    if (rule.greedy) {
        if (tid == 0)
            s.found = INT_MAX;
        __syncthreads();
        if (sm == r.m)
            atomicMin(&s.found, a.s_arg[slice0 + tid]);
        __syncthreads();
        if (tid == 0) {
            a.token[r.b] = s.found;
            if (a.logprob)
                a.logprob[r.b] = 0.0f;
        }
        return true;
    }
    r.E = rint(scaled(r.m, r.c));
    if (rule.by_k || rule.by_p || rule.by_min)
        return false;
    // the slices' masses in the row's unit
    const double d = sm > -INFINITY ? r.E - rint(scaled(sm, r.c)) : 64.0;
    const u64 shifted = d < 64.0 ? mass >> (int)d : 0;
    u64 base, Z, target;
    int slice = first_reaching<kThreads, 1>(s, a.slices, &base, &Z, &target, [&](int) { return shifted; },
                                              [&](u64 total) { return draw_target(r.u, total); });
    slice = min(slice, a.slices - 1);
    const double run_E = rint(scaled(a.s_max[slice0 + slice], r.c));
    draw_inside<kThreads>(a, r, row, s, slice * a.slice_len, a.slice_len, (target - 1 - base) << (int)(r.E - run_E), Z,
                          [&](int i) -> u64 {
                              return weight(scaled(one_logit(row, i), r.c), run_E);
                          });
    return true;
}

// Draws the rows that need no filter, and finds out where the others' filters
// end: the logits from `hi` on are kept by them, those in [lo, hi) are the
// candidates among which a filter ends.
template <typename T>
__global__ __launch_bounds__(kPlanThreads) void sample_plan_kernel(SampleParams a) {
    __shared__ PlanLds s;
    const int tid = threadIdx.x;
    Row r;
    r.b = blockIdx.x;
    const RowRule rule = row_rule(a, r.b);
    const size_t slice0 = (size_t)r.b * a.slices;
    RowPlan plan;
    plan.state = kDrawn;
    if (draw_unfiltered<kPlanThreads>(a, rule, r, static_cast<const T *>(a.logits) + (int64_t)r.b * a.row_stride, s)) {
        if (tid == 0)
            a.plan[r.b] = plan;
        return;
    }
    const double c = r.c, top = scaled(r.m, c);
    plan.state = kListed;
    plan.m = r.m;
    plan.lo = plan.hi = -FLT_MAX;
    plan.want = 0;
    plan.by_count = plan.then_p = plan.summed = false;
    plan.n = 0;
    if (rule.by_min)
        plan.lo = plan.hi = min_p_edge(rule, r.m);
    if (rule.by_k || rule.by_p) {
        // the slices' bins on the row's grid: a thread takes one bin of every
        // kGroups-th slice
        constexpr int kGroups = kPlanThreads / kBins, kAhead = 4;
        const int own = tid % kBins, group = tid / kBins;
        if (tid < kBins) {
            s.bin_count[tid] = 0;
            s.bin_mass[tid] = 0;
        }
        if (tid < a.slices) {   // how far a slice's grid and unit lie below the row's
            const double stop = scaled(a.s_max[slice0 + tid], c);
            s.bins_off[tid] = (int)fmin(floor(top * kBinsPerOctave) - floor(stop * kBinsPerOctave), (double)kBins);
            s.shift[tid] = (int)fmin(r.E - rint(stop), 63.0);
        }
        __syncthreads();
        const double top_bin = floor(top * kBinsPerOctave);
        for (int i0 = group; i0 < a.slices; i0 += kAhead * kGroups) {
            uint32_t n[kAhead];
            u64 mass[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const size_t at = (slice0 + min(i0 + k * kGroups, a.slices - 1)) * kBins + own;
                n[k] = rule.by_k ? a.h_count[at] : 0;
                mass[k] = rule.by_p ? a.h_mass[at] : 0;
            }
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const int i = i0 + k * kGroups;
                if (i >= a.slices)
                    continue;
                const int at = min(s.bins_off[i] + own, kBins - 1);
                if (n[k])
                    atomicAdd(&s.bin_count[at], n[k]);
                if (mass[k])
                    atomicAdd(&s.bin_mass[at], mass[k] >> s.shift[i]);
            }
        }
        __syncthreads();
        // How many logits a bin holds: counted for top-k, else at most its mass
        // over the weight at its lower edge, about a tenth too many (a weight
        // is up to two units short, and each slice's sum was rounded down).
        // The last bin has no lower edge and may hold any number.
        u64 count = 0;
        if (tid < kBins && rule.by_k) {
            count = s.bin_count[tid];
        } else if (tid < kBins - 1) {
            const double least = exp2((top_bin - tid) / kBinsPerOctave - r.E + 42.0) - 2.0;   // 2^9 at least
            count = s.bin_mass[tid] ? (u64)ceil((double)(s.bin_mass[tid] + (u64)a.slices) / least) : 0;
        } else if (tid == kBins - 1) {
            count = (u64)a.V;
        }
        u64 above, all, want, unused;
        int bin = kBins;   // the bin in which the first filter ends
        if (rule.by_k) {
            bin = first_reaching<kPlanThreads, 1>(s, kBins, &above, &all, &want, [&](int) { return count; },
                                                  [&](u64) { return (u64)rule.k; });
            plan.by_count = bin < kBins;   // else the row has no more usable logits than k
        }
        if (!plan.by_count && rule.by_p)
            bin = min(first_reaching<kPlanThreads, 1>(s, kBins, &above, &all, &want, [&](int i) { return s.bin_mass[i]; },
                                                      [&](u64 total) { return p_target(rule, total); }),
                      kBins - 1);
        if (bin < kBins) {
            plan.then_p = plan.by_count && rule.by_p;
            // logits down to the bin, and in it (thread bin holds both)
            const u64 down_to = block_scan<kPlanThreads / kWave>(count, s.waves, &unused);
            if (tid == bin) {
                s.n_low = down_to;
                s.n_bin = count;
            }
            __syncthreads();
            const u64 n_low = s.n_low, n_bin = s.n_bin;
            plan.lo = bin_edge(top_bin, bin, c);
            plan.hi = INFINITY;
            plan.want = want;
            // Only the bin's own logits become candidates where all down to it
            // are too many for the list, or too many to be compared pair by pair
            // while the bins hold the mass of those above.
            const bool sums = rule.by_p && !rule.by_min;
            if (n_low > kList || (n_low > kFew && sums && !plan.then_p)) {
                if (!plan.then_p) {
                    plan.hi = bin > 0 ? bin_edge(top_bin, bin - 1, c) : INFINITY;
                    plan.want = want - above;
                }
                plan.state = !plan.then_p && n_bin <= kList ? kListed : kScanned;
            }
            // What is kept anyway of each slice: where the bins hold masses and
            // no min-p takes part, their sum above the last bin.
            if (plan.state == kListed && sums) {
                plan.summed = true;
                const bool whole = plan.hi == INFINITY;
                for (int i = tid / kWave; i < a.slices; i += kPlanThreads / kWave) {
                    const int mine = whole ? 0 : bin - s.bins_off[i];   // bins of this slice that lie above it
                    u64 sum = 0;
                    for (int k = tid % kWave; k < mine; k += kWave)
                        sum += a.h_mass[(slice0 + i) * kBins + k];
                    sum = wave_incl_scan((uint64_t)sum);
                    if (tid % kWave == kWave - 1)
                        a.s_mass[slice0 + i] = sum >> s.shift[i];
                }
            }
        }
    }
    if (tid == 0)
        a.plan[r.b] = plan;
}

// Spreads the filtered rows over the chip a second time: appends each row's
// candidates to its list and sums the weights of what is kept anyway.
template <typename T, int kPasses>
__global__ __launch_bounds__(kSliceThreads) void sample_gather_kernel(SampleParams a) {
    constexpr int kVec = 16 / sizeof(T), kLoads = 16 * kPasses / kVec;
    __shared__ u64 waves[kSliceThreads / kWave];
    __shared__ int at_list;
    __shared__ float dense[kSliceUnit];
    const int b = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const int tid = threadIdx.x;
    const RowPlan &plan = a.plan[b];
    if (plan.state != kListed)
        return;
    const float lo = plan.lo, hi = plan.hi, m = plan.m;
    const size_t at_slice = (size_t)b * a.slices + slice;
    if (a.s_max[at_slice] < lo) {   // nothing here
        if (tid == 0)
            a.s_mass[at_slice] = 0;
        return;
    }
    const RowRule rule = row_rule(a, b);
    const int first = slice * a.slice_len, n = min(a.V - first, a.slice_len);
    const T *src = static_cast<const T *>(a.logits) + (int64_t)b * a.row_stride + first;
    float l[kLoads][kVec];
    load_slice<T, kPasses>(src, n, l);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kLoads; i++)
#pragma unroll
        for (int e = 0; e < kVec; e++)
            mine += l[i][e] >= lo && l[i][e] < hi;
    if (!plan.summed) {
        u64 total = 0;
        if (hi < INFINITY) {
            // The logits to be summed are put side by side first, a pass at a
            // time: a weight costs a wavefront the same for one lane as for all
            // (a min-p that keeps 5 % took 39 us in place).
            const double E = rint(scaled(m, rule.c));
            u64 sum = 0;
#pragma unroll
            for (int pass = 0; pass < kPasses; pass++) {
                int kept = 0;
#pragma unroll
                for (int i = pass * kLoads / kPasses; i < (pass + 1) * kLoads / kPasses; i++)
#pragma unroll
                    for (int e = 0; e < kVec; e++)
                        kept += l[i][e] >= hi;
                u64 n;   // (the scan's barriers end the reads of the pass before)
                int at = (int)block_scan<kSliceThreads / kWave>((u64)kept, waves, &n) - kept;
                if (kept) {
#pragma unroll
                    for (int i = pass * kLoads / kPasses; i < (pass + 1) * kLoads / kPasses; i++)
#pragma unroll
                        for (int e = 0; e < kVec; e++)
                            if (l[i][e] >= hi)
                                dense[at++] = l[i][e];
                }
                __syncthreads();
                for (int i = tid; i < (int)n; i += kSliceThreads)
                    sum += passes_min(rule, dense[i], m) ? weight(scaled(dense[i], rule.c), E) : 0;
            }
            block_scan<kSliceThreads / kWave>(sum, waves, &total);
        }
        if (tid == 0)
            a.s_mass[at_slice] = total;
    }
    u64 all;
    int at = (int)block_scan<kSliceThreads / kWave>((u64)mine, waves, &all) - mine;
    if (all == 0)
        return;
    if (tid == 0)
        at_list = atomicAdd(&a.plan[b].n, (int)all);
    __syncthreads();
    at += at_list;
    if (mine == 0)
        return;
#pragma unroll
    for (int i = 0; i < kLoads; i++)
#pragma unroll
        for (int e = 0; e < kVec; e++)
            if (l[i][e] >= lo && l[i][e] < hi) {
                if (at < a.list_len)   // (the bins counted no more)
                    a.list[(size_t)b * a.list_len + at] = rank_of(l[i][e], first + (i * kSliceThreads + tid) * kVec + e);
                at++;
            }
}

template <typename T>
__global__ __launch_bounds__(kFilterThreads) void sample_filter_kernel(SampleParams a) {
    extern __shared__ u64 pick_lds[];
    FilterLds &s = *reinterpret_cast<FilterLds *>(pick_lds);
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    Row r;
    r.b = blockIdx.x;
    const RowPlan plan = a.plan[r.b];
    if (plan.state == kDrawn)
        return;
    const RowRule rule = row_rule(a, r.b);
    const size_t slice0 = (size_t)r.b * a.slices;
    const T *row = static_cast<const T *>(a.logits) + (int64_t)r.b * a.row_stride;
    r.u = clamp_u(a.u[r.b]);
    r.m = plan.m;
    r.c = rule.c;
    r.E = rint(scaled(r.m, r.c));
    const bool listed = plan.state == kListed;
    const int n_list = listed ? min(plan.n, a.list_len) : 0;
    if (tid < a.slices)
        s.slice[tid] = listed ? a.s_mass[slice0 + tid] : 0;
    __syncthreads();

    const auto weight_of = [&](float l) { return weight(scaled(l, r.c), r.E); };
    const auto logit_of = [](u64 rank) { return from_order_bits((uint32_t)(rank >> kMaxVocabBits)); };
    constexpr int kIndex = (1 << kMaxVocabBits) - 1;
    const auto index_of = [](u64 rank) { return kIndex - (int)(rank & kIndex); };
    u64 all;
    for (int i = tid; i < n_list; i += kFilterThreads) {
        const u64 rank = a.list[(size_t)r.b * a.list_len + i];
        s.list[i] = rank;
        s.weight[i] = weight_of(logit_of(rank));
    }
    __syncthreads();

    if (listed && plan.hi == INFINITY && n_list <= kFew) {
        // Few logits in question: each is compared with all the others, by kEach
        // neighbouring lanes.
        const int own = tid / kEach, part = tid % kEach;
        const bool mine = own < n_list;
        const u64 rank = mine ? s.list[own] : 0, w = mine ? s.weight[own] : 0;
        u64 in_front = 0, mass_in_front = 0;
        if (mine)
            for (int j = part; j < n_list; j += kEach) {
                const bool first = s.list[j] > rank;
                in_front += first;
                mass_in_front += first ? s.weight[j] : 0;
            }
        in_front = sum_each(in_front);
        mass_in_front = sum_each(mass_in_front);
        bool kept = mine && !(plan.by_count && in_front >= (u64)rule.k);
        if (rule.by_p) {
            u64 want = plan.want;   // without top-k, of the whole row's mass
            if (plan.by_count) {
                block_scan<kFilterThreads / kWave>(kept && part == 0 ? w : 0, s.waves, &all);
                want = p_target(rule, all);
            }
            kept = kept && mass_in_front < want;
        }
        kept = kept && passes_min(rule, logit_of(rank), r.m);
        u64 Z;
        block_scan<kFilterThreads / kWave>(kept && part == 0 ? w : 0, s.waves, &Z);   // (its barriers order the loops' reads)
        if (mine && part == 0)
            s.weight[own] = kept ? w : 0;
        __syncthreads();
        u64 target, unused, before = 0;
        fraction_of(r.u, Z, &target, &unused);
        if (kept)   // (the same for all lanes of a logit)
            for (int j = part; j < n_list; j += kEach)
                before += index_of(s.list[j]) < index_of(rank) ? s.weight[j] : 0;
        before = sum_each(before);
        if (kept && part == 0 && before <= target && target < before + w)
            write_token(a, r, index_of(rank), logit_of(rank), Z);
        return;
    }

    u64 cut = 0;   // lowest rank that is kept
    if (plan.want) {
        // Finds the rank at which the running sum (of counts, or of weights) of
        // the candidates reaches `want`, from its highest digit down until few
        // candidates share the digits found, which are compared pair by pair;
        // for a top-p of what a top-k keeps, once more with the weights.
        // Candidates that do not fit a list are read from the row.
        const auto for_candidates = [&](auto f) {
            if (listed) {
                for (int i = tid; i < n_list; i += kFilterThreads)
                    f(s.list[i], [&] { return s.weight[i]; });
            } else {
                for_row(row, a.V, [&](int, const float(&l)[4], int at) {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (l[e] >= plan.lo && l[e] < plan.hi)
                            f(rank_of(l[e], at + e), [&] { return weight_of(l[e]); });
                });
            }
        };
        // the highest bit in which candidates differ
        int top = 32 + kMaxVocabBits;
        u64 same = 0;
        if (listed) {
            if (tid == 0)
                s.differ = 0;
            __syncthreads();
            same = s.list[0];
            u64 differ = 0;
            for (int i = tid; i < n_list; i += kFilterThreads)
                differ |= s.list[i] ^ same;
#pragma unroll
            for (int d = 32; d; d >>= 1)
                differ |= __shfl_xor(differ, d, kWave);
            if (lane == 0 && differ)
                atomicOr(&s.differ, differ);
            __syncthreads();
            top = s.differ ? 64 - __clzll((long long)s.differ) : 0;
        }
        bool counts = plan.by_count;
        u64 want = plan.want;
        for (int round = 0; round <= (int)plan.then_p; round++) {
            u64 prefix = top < 64 ? same >> top : 0;
            const u64 floor_rank = cut;
            int shift = top;
            while (shift > 0) {
                if (!listed || n_list > kFew) {
                    const int next = max(shift - kDigitBits, 0), digits = 1 << (shift - next);
                    for (int i = tid; i < kDigits; i += kFilterThreads)
                        s.digit[i] = 0;
                    if (tid == 0)
                        s.n = 0;
                    __syncthreads();
                    for_candidates([&](u64 rank, auto weight) {
                        if (rank >> shift == prefix && rank >= floor_rank)
                            atomicAdd(&s.digit[digits - 1 - ((rank >> next) & (digits - 1))], counts ? 1ull : weight());
                    });
                    __syncthreads();
                    u64 in_front, sum, goal;
                    // (a target past the sum, by rounding of the bins' masses, takes the last one)
                    int d = first_reaching<kFilterThreads, kDigits / kFilterThreads>(
                        s, digits, &in_front, &sum, &goal, [&](int i) { return s.digit[i]; },
                        [&](u64 sum) { return want < sum ? want : sum; });
                    d = min(d, digits - 1);
                    want = goal - in_front;
                    prefix = prefix << (shift - next) | (u64)(digits - 1 - d);
                    shift = next;
                    if (shift == 0)
                        break;
                } else {
                    if (tid == 0)
                        s.n = 0;
                    __syncthreads();
                }
                for_candidates([&](u64 rank, auto weight) {
                    if (rank >> shift == prefix && rank >= floor_rank) {
                        const int i = atomicAdd(&s.n, 1);
                        if (i < kFew) {
                            s.few[i] = rank;
                            s.few_weight[i] = counts ? 1 : weight();
                        }
                    }
                });
                if (tid == 0)
                    s.cut = max(prefix << shift, floor_rank);   // (all of them, should rounding leave the target out of reach)
                __syncthreads();
                if (s.n <= kFew) {
                    const int own = tid / kEach, n = s.n;
                    const bool mine = own < n;
                    u64 before = 0;
                    if (mine)
                        for (int j = tid % kEach; j < n; j += kEach)
                            before += s.few[j] > s.few[own] ? s.few_weight[j] : 0;
                    before = sum_each(before);
                    if (mine && before < want && before + s.few_weight[own] >= want)
                        s.cut = s.few[own];
                    __syncthreads();
                    prefix = s.cut;
                    break;
                }
                __syncthreads();
            }
            cut = prefix;
            if (plan.then_p && round == 0) {
                u64 kept = 0;
                for_candidates([&](u64 rank, auto weight) { kept += rank >= cut ? weight() : 0; });
                block_scan<kFilterThreads / kWave>(kept, s.waves, &all);
                want = p_target(rule, all);
                counts = false;
            }
        }
    }

    // the kept mass of every slice, and the draw
    if (listed) {
        // (a slice's candidates are neighbours in the list: most wavefronts have
        // one slice, whose sum takes one addition in place of 64 to one address)
        for (int i0 = 0; i0 < n_list; i0 += kFilterThreads) {
            const int i = i0 + tid;
            const u64 rank = s.list[min(i, n_list - 1)];
            const u64 w = i < n_list && rank >= cut && passes_min(rule, logit_of(rank), r.m) ? s.weight[i] : 0;
            const int slice = index_of(rank) / a.slice_len;
            if (__all(slice == first_lane_int(slice))) {
                const u64 sum = wave_incl_scan((uint64_t)w);
                if (lane == kWave - 1 && sum)
                    atomicAdd(&s.slice[slice], sum);
            } else if (w) {
                atomicAdd(&s.slice[slice], w);
            }
        }
    } else {
        for_row(row, a.V, [&](int run, const float(&l)[4], int at) {
            u64 sum = 0;
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (l[e] >= plan.lo && rank_of(l[e], at + e) >= cut && passes_min(rule, l[e], r.m))
                    sum += weight_of(l[e]);
            sum = wave_incl_scan((uint64_t)sum);
            if (lane == kWave - 1 && sum)
                atomicAdd(&s.slice[run * kRun / a.slice_len], sum);
        });
    }
    __syncthreads();
    u64 Z, target, base;
    int slice = first_reaching<kFilterThreads, 1>(s, a.slices, &base, &Z, &target, [&](int i) { return s.slice[i]; },
                                                  [&](u64 total) { return draw_target(r.u, total); });
    slice = min(slice, a.slices - 1);
    draw_inside<kFilterThreads>(a, r, row, s, slice * a.slice_len, a.slice_len, target - 1 - base, Z, [&](int i) -> u64 {
        const float l = one_logit(row, i);
        return l >= plan.lo && rank_of(l, i) >= cut && passes_min(rule, l, r.m) ? weight_of(l) : 0;
    });
}

struct SamplePlan {
    int slices, slice_len;
    size_t arg_off, mass_off, count_off, hmass_off, plan_off, list_off, bytes;
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
    pl->plan_off = pl->hmass_off + up(n * kBins * sizeof(u64));
    pl->list_off = pl->plan_off + up(B * sizeof(RowPlan));
    pl->bytes = pl->list_off + up((size_t)B * std::min(kList, V) * sizeof(u64));
    return TS_OK;
}

template <typename T, int kPasses>
hipError_t launch_sample(const SampleParams &a, int B, hipStream_t hs) {
    const unsigned rows = (unsigned)B, slices = rows * (unsigned)a.slices;
    hipError_t e;
    hipLaunchKernelGGL((sample_slices_kernel<T, kPasses>), dim3(slices), dim3(kSliceThreads), 0, hs, a);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    hipLaunchKernelGGL(sample_plan_kernel<T>, dim3(rows), dim3(kPlanThreads), 0, hs, a);
    if ((e = hipGetLastError()) != hipSuccess || !(a.top_k || a.top_p || a.min_p))
        return e;
    hipLaunchKernelGGL((sample_gather_kernel<T, kPasses>), dim3(slices), dim3(kSliceThreads), 0, hs, a);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    hipLaunchKernelGGL(sample_filter_kernel<T>, dim3(rows), dim3(kFilterThreads), sizeof(FilterLds), hs, a);
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
    a.plan = reinterpret_cast<RowPlan *>(ws + pl.plan_off);
    a.list = reinterpret_cast<u64 *>(ws + pl.list_off);
    a.list_len = std::min(kList, vocab);
    a.row_stride = row_stride;
    a.V = vocab;
    a.slices = pl.slices;
    a.slice_len = pl.slice_len;
    hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    const bool f32 = logits_type == TS_LOGITS_F32, shorter = pl.slice_len == kSliceUnit;
    const hipError_t e = f32 ? (shorter ? launch_sample<float, 1>(a, num_seqs, hs) : launch_sample<float, kLongSlice>(a, num_seqs, hs))
                             : (shorter ? launch_sample<uint16_t, 1>(a, num_seqs, hs)
                                        : launch_sample<uint16_t, kLongSlice>(a, num_seqs, hs));
    return e == hipSuccess ? TS_OK : hip_fail(e, "sampling launch");
}

}  // extern "C"
