// logit_rules.hip -- what a request asks of its logits before the draw: penalties
// for tokens that its text holds already, biases, and a grammar's mask.
//
// For token v of a row with logit l, with n the number of times that v is among
// the row's answer (its tokens behind the prompt) and "seen" if it is among its
// tokens at all, in float32 and in this order:
//   x = l;  seen: x = x > 0 ? x * (1 / repetition) : x * repetition;
//   n > 0: x -= frequency * n + presence;  biased: x += the sum of v's biases;
//   not allowed: x = -inf;  out = x, rounded once.
//
// A workgroup takes kSlice tokens of the vocabulary of one row, eight to a thread.
// It counts the row's tokens that fall into its slice in LDS (integers, so the
// order of the additions does not matter), reading all of the row's tokens: rows
// have few thousands of them, and the slices of a row are neighbours on one XCD,
// whose L2 holds them.  Its logits are on their way meanwhile.  Biases are added up
// in LDS too, in the order of the list whatever threads they fall to: of the
// threads that hold biases of one token, the first adds its own, then the next
// (three barriers for each, so a list that names one token over and over takes time
// for every mention).
// One launch (of shapes with 2^23 slices and more, another for the rows behind those
// that fill one), nothing kept in memory between slices or calls.
//
// In place, a thread that has nothing to change neither reads nor writes its eight
// logits; one that has rewrites all of them.
//
// What bounds it.  Many rows: vector instructions, 89 % busy, and the bytes.  200 rows of
// 151,936 bf16 logits, masks, biases and texts of 4,000 tokens on average take 38.5 us
// (the bytes alone need 26): 133 instructions for a wavefront's 512 tokens of the
// vocabulary and about as many for the text, the biases and addresses.  What mattered
// is that no load waits for another: logits and masks stay as they are in memory until
// the text is counted (45.6 -> 42.4), a row's numbers are loaded together (41.8), and
// no lane's load of logits is masked off, which made the compiler wait for it to move
// registers (38.5).  Before these, when it took 45 us, slices of 8,192 tokens on 1,024
// threads took 47 us, on 512 threads 47, 4,096 on 256 threads 50; workgroups that keep
// a row's text for several slices 49; working out only the tokens of the text, whoever
// finds their count, is a longer chain (77); none was measured again since.  In place,
// with masks on two rows of three, it takes as long (43 against 42 us in one loop).  Few
// rows: the chain lengths -> tokens -> LDS -> stores (8 rows 8 us in a graph, about the
// call from Python).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "ts_attn.h"
#include "ts_internal.h"

namespace tsattn {

namespace {

constexpr int kThreads = 512;
constexpr int kMostGroups = (1 << 23) - 1;     // of a launch, which has less than 2^32 threads
constexpr int kPer = 8;                        // tokens of a thread
constexpr int kSlice = kThreads * kPer;
constexpr int kAhead = 4;                      // groups of four text tokens whose loads are in flight together
constexpr int kTable = kSlice + kWave;          // and a place for each lane's tokens of other slices
constexpr uint32_t kInPrompt = 0x80000000u;
constexpr uint32_t kNone = 0x80000000u;         // no bias: -0, which added changes nothing, +0 and -0 neither

struct RulesParams {
    const void *logits;
    void *out;
    const int32_t *tokens;
    // A row's numbers, each an array with an entry for each row whatever is given
    // (`has`), so that they are loaded together; all NULL if nothing of them is.
    const int32_t *lens, *prompt_lens, *bias_starts;
    const float *repetition, *frequency, *presence;
    const int32_t *bias_tokens;
    const float *bias_values;
    const uint32_t *allowed;
    int64_t row_stride, out_stride, token_stride, allowed_stride;
    int first_row, vocab, slices, max_tokens, num_biases;
    bool in_place;
    uint8_t has;
};
constexpr int kHasPrompt = 1, kHasRepetition = 2, kHasFrequency = 4, kHasPresence = 8;

// Loads and stores of any element alignment.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Many {
    T x[N];
};

// A thread's eight logits as they are in memory.  Nothing is done with them until
// load8_rest, so that the loads behind theirs do not wait for them.
template <typename T>
struct Raw8 {
    uint32_t w[kPer * sizeof(T) / 4];
    __device__ __forceinline__ float value(int e) const {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[e]);
        else
            return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
    }
};
template <typename T>
__device__ __forceinline__ void load8(const T *src, int n, Raw8<T> &r) {
    if (n >= kPer)
        __builtin_memcpy(&r, reinterpret_cast<const Many<T, kPer> *>(src), sizeof r);
}
// Those of a row's last thread, if it has fewer.
template <typename T>
__device__ __forceinline__ void load8_rest(const T *src, int n, Raw8<T> &r) {
    if (n <= 0 || n >= kPer)
        return;
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
    Bits x[kPer];
#pragma unroll
    for (int e = 0; e < kPer; e++)
        x[e] = reinterpret_cast<const Bits *>(src)[min(e, n - 1)];
#pragma unroll
    for (int i = 0; i < (int)(sizeof r / 4); i++) {
        if constexpr (sizeof(T) == 4)
            r.w[i] = x[i];
        else
            r.w[i] = (uint32_t)x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
    }
}
__device__ __forceinline__ void store8(float *dst, int n, const float x[kPer]) {
    if (n >= kPer) {
        Many<float, kPer> v;
#pragma unroll
        for (int e = 0; e < kPer; e++)
            v.x[e] = x[e];
        *reinterpret_cast<Many<float, kPer> *>(dst) = v;
    } else {
#pragma unroll
        for (int e = 0; e < kPer; e++)
            if (e < n)
                dst[e] = x[e];
    }
}
__device__ __forceinline__ void store8(uint16_t *dst, int n, const float x[kPer]) {
    Many<uint32_t, kPer / 2> v;
#pragma unroll
    for (int e = 0; e < kPer; e += 2)
        v.x[e / 2] = pack_bf16x2(x[e], x[e + 1]);
    if (n >= kPer) {
        __builtin_memcpy(dst, &v, sizeof v);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; e++)
            if (e < n)
                dst[e] = (uint16_t)(v.x[e / 2] >> 16 * (e % 2));
    }
}

// A barrier for what is in LDS: loads from memory stay under way.
__device__ __forceinline__ void lds_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A penalty, or `off` where it is not given or not finite.
__device__ __forceinline__ float penalty(bool given, float x, float off) { return given && fabsf(x) < INFINITY ? x : off; }

template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void logit_rules_kernel(RulesParams p) {
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    uint32_t *const count = lds;                              // [kSlice] times in the answer; kInPrompt
    float *const bias = reinterpret_cast<float *>(lds + kTable);   // [kSlice], where there are biases
    __shared__ int s_pending;
    const int at = xcd_worker(blockIdx.x, gridDim.x);
    const int b = p.first_row + at / p.slices, base = at % p.slices * kSlice, tid = threadIdx.x;
    const int n = p.vocab - base - kPer * tid;                // of this thread's tokens exist
    const TI *const src = static_cast<const TI *>(p.logits) + b * p.row_stride + base + kPer * tid;
    TO *const dst = static_cast<TO *>(p.out) + b * p.out_stride + base + kPer * tid;
    const uint32_t here = (uint32_t)min(kSlice, p.vocab - base);   // tokens of the slice
    // Lengths, then every first load, before anything waits for one.
    int first = 0, end = 0, len = 0, prompt = 0;
    float rep = 1.0f, freq = 0.0f, pres = 0.0f;
    if (p.lens) {
        const auto number = [&](const float *x) { return __int_as_float(ld_meta(reinterpret_cast<const int32_t *>(x), b)); };
        const int bias_first = ld_meta(p.bias_starts, b), bias_end = ld_meta(p.bias_starts, p.bias_tokens ? b + 1 : b);
        const int text_len = ld_meta(p.lens, b), prompt_len = ld_meta(p.prompt_lens, b);
        const float r = number(p.repetition), f = number(p.frequency), q = number(p.presence);
        first = p.bias_tokens ? bias_first : 0;
        end = p.bias_tokens ? bias_end : 0;
        len = p.tokens ? text_len : 0;
        prompt = p.has & kHasPrompt ? prompt_len : 0;
        rep = penalty(p.has & kHasRepetition, r, 1.0f);
        rep = rep > 0.0f ? rep : 1.0f;
        freq = penalty(p.has & kHasFrequency, f, 0.0f);
        pres = penalty(p.has & kHasPresence, q, 0.0f);
    }
    // (Threads without eight logits read the row's first ones: no lane is masked.)
    Raw8<TI> raw;
    if (!p.in_place && p.vocab >= kPer)
        load8(n >= kPer ? src : src - (base + kPer * tid), kPer, raw);
    uint32_t open = ~0u;                                      // the mask's word of this thread's tokens
    if (p.allowed && n > 0)
        open = p.allowed[b * p.allowed_stride + (base + kPer * tid) / 32];
    first = min(max(first, 0), p.num_biases);
    end = min(max(end, 0), p.num_biases);
    len = min(max(len, 0), p.max_tokens);
    prompt = min(max(prompt, 0), len);
    int32_t bias_token = 0;                                   // the bias that this thread holds, if there is one
    float bias_w = 0.0f;
    const auto load_bias = [&](int j0) {
        if (j0 + tid < end) {
            bias_token = p.bias_tokens[j0 + tid];
            bias_w = p.bias_values[j0 + tid];
        }
    };
    if (first < end)
        load_bias(first);
    const int32_t *const text = p.tokens + (p.tokens ? b * p.token_stride : 0);
    const int whole = len / 4 * 4;
    Many<int32_t, 4> ids[kAhead];
    // Groups of four tokens from i0 on, -1 where the text has none (the conditions on
    // whole wavefronts are scalar).
    const int lane4 = 4 * (tid % kWave), wave4 = first_lane_int(4 * (tid - tid % kWave));
    const auto load_text = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            const int at = i0 + wave4 + 4 * kThreads * k;
            ids[k] = Many<int32_t, 4>{{-1, -1, -1, -1}};
            if (at < whole && at + lane4 < whole)
                ids[k] = *reinterpret_cast<const Many<int32_t, 4> *>(text + at + lane4);
        }
    };
    load_text(0);
    int32_t odd = -1;                                         // the last tokens
    if (whole + tid < len)
        odd = text[whole + tid];
    if (!p.in_place)
        load8_rest(src, n, raw);

    u32x4_t *const zero = reinterpret_cast<u32x4_t *>(lds);
#pragma unroll
    for (int i = 0; i < kSlice / 4 / kThreads; i++) {
        zero[i * kThreads + tid] = u32x4_t{0u, 0u, 0u, 0u};
        if (p.bias_tokens)
            zero[kTable / 4 + i * kThreads + tid] = u32x4_t{kNone, kNone, kNone, kNone};
    }
    lds_sync();

    for (int j0 = first; j0 < end; j0 += kThreads) {
        const uint32_t bias_at = (uint32_t)bias_token - (uint32_t)base;   // its place in the slice
        bool pending = j0 + tid < end && bias_at < here;
        const uint32_t mine = kThreads - tid;             // the first thread has the largest
        for (;;) {
            if (tid == 0)
                s_pending = 0;
            if (pending)
                atomicMax(&count[bias_at], mine);
            lds_sync();
            const bool turn = pending && count[bias_at] == mine;
            if (pending && !turn)
                s_pending = 1;
            lds_sync();
            if (turn) {
                bias[bias_at] += bias_w;
                count[bias_at] = 0;
                pending = false;
            }
            const int more = s_pending;
            lds_sync();
            if (!more)
                break;
        }
        if (j0 + kThreads < end)
            load_bias(j0 + kThreads);
    }

    if (p.tokens) {
        // No branches: a token of another slice goes to a place of the lane's own.
        const uint32_t aside = kSlice + tid % kWave;
        const auto place = [&](int32_t token, bool counts) {
            const uint32_t t = (uint32_t)token - (uint32_t)base;
            return counts && t < here ? t : aside;
        };
        for (int i0 = 0; i0 < whole; i0 += 4 * kThreads * kAhead) {
            if (i0 > 0)
                load_text(i0);
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const int at = i0 + wave4 + 4 * kThreads * k;
                if (at >= whole)
                    break;
                if (at >= prompt) {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        atomicAdd(&count[place(ids[k].x[e], true)], 1u);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        atomicOr(&count[place(ids[k].x[e], at + lane4 + e < prompt)], kInPrompt);
                    if (at + 4 * kWave > prompt)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            atomicAdd(&count[place(ids[k].x[e], at + lane4 + e >= prompt)], 1u);
                }
            }
        }
        if (tid < 4) {
            atomicOr(&count[place(odd, whole + tid < prompt)], kInPrompt);
            atomicAdd(&count[place(odd, whole + tid >= prompt)], 1u);
        }
        lds_sync();
    }
    if (n <= 0)
        return;
    uint32_t c[kPer];
    float w[kPer];
    asm volatile("" : "+v"(open));                            // (or it would be turned round where it is loaded, and waited for)
    const uint32_t closed = ~open >> (base + kPer * tid) % 32 & ((1u << kPer) - 1);   // bit e: token e is not allowed
    bool any = closed != 0;
#pragma unroll
    for (int e = 0; e < kPer; e += 4) {
        const u32x4_t cv = *reinterpret_cast<const u32x4_t *>(count + kPer * tid + e);
        f32x4_t wv = {-0.0f, -0.0f, -0.0f, -0.0f};
        if (p.bias_tokens)
            wv = *reinterpret_cast<const f32x4_t *>(bias + kPer * tid + e);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            c[e + i] = cv[i];
            w[e + i] = wv[i];
            any |= cv[i] != 0 || wv[i] != 0.0f;   // (NaN differs from 0)
        }
    }
    if (p.in_place) {
        if (!any)
            return;
        load8(src, n, raw);
        load8_rest(src, n, raw);
    }
    // (Without branches, which some token of a wavefront's 512 would mostly take.)
    const float inverse = 1.0f / rep;
    float x[kPer];
#pragma unroll
    for (int e = 0; e < kPer; e++) {
        x[e] = raw.value(e);
        const uint32_t times = c[e] & ~kInPrompt;
        x[e] *= c[e] ? x[e] > 0.0f ? inverse : rep : 1.0f;
        x[e] -= times ? freq * (float)times + pres : 0.0f;
        x[e] += w[e];
        x[e] = closed >> e & 1 ? -INFINITY : x[e];
    }
    store8(dst, n, x);
}

}  // namespace

}  // namespace tsattn

using namespace tsattn;

extern "C" {

int ts_logit_rules(const ts_rules_config *cfg, const void *logits, void *out, const int32_t *tokens,
                   const int32_t *lens, const int32_t *prompt_lens, const float *repetition, const float *frequency,
                   const float *presence, const int32_t *bias_starts, const int32_t *bias_tokens,
                   const float *bias_values, const uint32_t *allowed, void *stream) {
    clear_error();
    if (!cfg || !logits || !out)
        return fail(TS_ERR_NULL, "a pointer is NULL");
    if (cfg->num_seqs < 1 || cfg->num_seqs > 65536)
        return fail(TS_ERR_SHAPE, "num_seqs %d outside [1, 65536]", cfg->num_seqs);
    if (cfg->vocab < 1 || cfg->vocab > (1 << 20))
        return fail(TS_ERR_SHAPE, "vocab %d outside [1, 2^20]", cfg->vocab);
    const auto known = [](int t) { return t == TS_LOGITS_F32 || t == TS_LOGITS_BF16; };
    if (!known(cfg->logits_type) || !known(cfg->out_type))
        return fail(TS_ERR_ARG, "logits_type %d or out_type %d unknown", cfg->logits_type, cfg->out_type);
    const int64_t most = 1LL << 40;
    if (cfg->row_stride < cfg->vocab || cfg->row_stride > most || cfg->out_stride < cfg->vocab || cfg->out_stride > most)
        return fail(TS_ERR_ARG, "row_stride %lld or out_stride %lld below vocab, or above 2^40", (long long)cfg->row_stride,
                    (long long)cfg->out_stride);
    const int in_size = cfg->logits_type == TS_LOGITS_F32 ? 4 : 2, out_size = cfg->out_type == TS_LOGITS_F32 ? 4 : 2;
    if ((uintptr_t)logits % in_size || (uintptr_t)out % out_size)
        return fail(TS_ERR_ARG, "misaligned logits or out");
    if (out == logits && (cfg->out_type != cfg->logits_type || cfg->out_stride != cfg->row_stride))
        return fail(TS_ERR_ARG, "out == logits needs one type and equal strides");
    const bool penalties = repetition || frequency || presence;
    if (!tokens && (penalties || lens || prompt_lens))
        return fail(TS_ERR_NULL, "penalties and lengths need tokens");
    if (tokens && !lens)
        return fail(TS_ERR_NULL, "tokens need lens");
    if (tokens && (cfg->max_tokens < 0 || cfg->max_tokens > (1 << 29) || cfg->token_stride < cfg->max_tokens ||
                   cfg->token_stride > most))
        return fail(TS_ERR_ARG, "max_tokens %d outside [0, 2^29], or token_stride %lld below it or above 2^40",
                    cfg->max_tokens, (long long)cfg->token_stride);
    if (!bias_starts != !bias_tokens || !bias_starts != !bias_values)
        return fail(TS_ERR_NULL, "biases need starts, tokens and values");
    if (bias_starts && (cfg->num_biases < 0 || cfg->num_biases > (1 << 30)))
        return fail(TS_ERR_ARG, "num_biases %d outside [0, 2^30]", cfg->num_biases);
    if (allowed && (cfg->allowed_stride < (cfg->vocab + 31) / 32 || cfg->allowed_stride > most))
        return fail(TS_ERR_ARG, "allowed_stride %lld below vocab / 32, or above 2^40", (long long)cfg->allowed_stride);
    if (((uintptr_t)tokens | (uintptr_t)lens | (uintptr_t)prompt_lens | (uintptr_t)repetition | (uintptr_t)frequency |
         (uintptr_t)presence | (uintptr_t)bias_starts | (uintptr_t)bias_tokens | (uintptr_t)bias_values | (uintptr_t)allowed) & 3)
        return fail(TS_ERR_ARG, "misaligned pointer (4 B needed)");
    int st = check_device();
    if (st)
        return st;
    RulesParams p;
    p.logits = logits;
    p.out = out;
    p.tokens = penalties && cfg->max_tokens > 0 ? tokens : nullptr;
    p.bias_tokens = bias_starts && cfg->num_biases > 0 ? bias_tokens : nullptr;
    const int32_t *const some = p.tokens ? lens : p.bias_tokens ? bias_starts : nullptr;
    p.lens = p.tokens ? lens : some;
    p.prompt_lens = p.tokens && prompt_lens ? prompt_lens : some;
    p.bias_starts = p.bias_tokens ? bias_starts : some;
    const auto given = [&](const float *x) { return p.tokens && x ? x : reinterpret_cast<const float *>(some); };
    p.repetition = given(repetition);
    p.frequency = given(frequency);
    p.presence = given(presence);
    p.has = (prompt_lens ? kHasPrompt : 0) | (repetition ? kHasRepetition : 0) | (frequency ? kHasFrequency : 0) |
            (presence ? kHasPresence : 0);
    p.bias_values = bias_values;
    p.allowed = allowed;
    p.row_stride = cfg->row_stride;
    p.out_stride = cfg->out_stride;
    p.token_stride = cfg->token_stride;
    p.allowed_stride = cfg->allowed_stride;
    p.vocab = cfg->vocab;
    p.slices = (cfg->vocab + kSlice - 1) / kSlice;
    p.max_tokens = cfg->max_tokens;
    p.num_biases = cfg->num_biases;
    p.in_place = out == logits;
    const bool f_in = cfg->logits_type == TS_LOGITS_F32, f_out = cfg->out_type == TS_LOGITS_F32;
    const auto kernel = f_in ? f_out ? logit_rules_kernel<float, float> : logit_rules_kernel<float, uint16_t>
                             : f_out ? logit_rules_kernel<uint16_t, float> : logit_rules_kernel<uint16_t, uint16_t>;
    const size_t lds = (kTable + (p.bias_tokens ? kSlice : 0)) * sizeof(uint32_t);
    const int row_step = kMostGroups / p.slices;   // rows of a launch
    for (p.first_row = 0; p.first_row < cfg->num_seqs; p.first_row += row_step) {
        const int rows = std::min(row_step, cfg->num_seqs - p.first_row);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * p.slices)), dim3(kThreads), lds, reinterpret_cast<hipStream_t>(stream), p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return hip_fail(e, "logit rules launch");
    }
    return TS_OK;
}

}  // extern "C"
