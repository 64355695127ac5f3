// rope_common.h -- pieces shared by the kernels that norm, rotate and append:
// a head's vector is held by head_dim / 8 neighbouring lanes, 8 values each.
#pragma once

#include "attn_common.h"
#include "ts_attn.h"

namespace tsattn {

// Checks of ts_rope_append and ts_rope_append_kv8 on what both are given; with
// no tokens (TS_OK) the pointers are not looked at.
int check_rope(const ts_chunk_shape *s, const ts_rope_config *cfg, const void *q, const void *k, const void *v,
               void *q_out, void *k_pages, void *v_pages, const int32_t *page_table, const int32_t *ctx_lens,
               const int32_t *q_starts, const float *inv_freq, const void *q_norm, const void *k_norm);

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

}  // namespace tsattn
