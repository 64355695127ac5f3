// attn_verify_kv8.hip -- paged decode and verify attention over the cache held in
// 8 bits (kv8_common.h): the wavefront-streams kernels of attn_verify.hip, with
// their partition, groups and merges, on half of the bytes.
//
// A step is two pages, so that a wavefront has as many bytes under way as with
// bf16 pages, and 32 keys fill one value product (16x16x32 instead of two
// 16x16x16).  Codes become bf16 in registers, two to an instruction that takes
// the page's power along, which is exact; scores, weights and sums are then those
// of the bf16 kernels.  Keys: a lane's 16 bytes of a row are its operands of two
// k-steps, so queries are loaded in that order of dims.  Values: two tokens'
// bytes are interleaved before the conversion, which then leaves pairs of tokens
// for a dim, the order of the value product's operand: 16 byte permutations
// instead of 32 for a step.
//
// What bounds it: bytes.  Matrix and vector instructions of a step take about a
// third of the time in which its 8 KiB arrive.
#include "attn_verify.h"

namespace tsattn {

typedef void (*kernel_fn)(AttnParams);

kernel_fn verify_group_kv8_variant(int D, int NB, int *lds_bytes) {
#define TS_VG(DD, NN)                                                      \
    if (D == DD && NB == NN) {                                             \
        *lds_bytes = (int)sizeof(typename Verify<DD, NN, true>::GroupLds); \
        return verify_group_kernel<DD, NN, true>;                          \
    }
    TS_VG(64, 1) TS_VG(64, 2) TS_VG(64, 3) TS_VG(64, 4) TS_VG(128, 1) TS_VG(128, 2)
#undef TS_VG
    return nullptr;
}

kernel_fn verify_kv8_variant(int D, int NB) {
#define TS_VF(DD, NN) \
    if (D == DD && NB == NN) return verify_kernel<DD, NN, true>;
    TS_VF(64, 1) TS_VF(64, 2) TS_VF(64, 3) TS_VF(64, 4)
    TS_VF(128, 1) TS_VF(128, 2) TS_VF(128, 3) TS_VF(128, 4)
#undef TS_VF
    return nullptr;
}

}  // namespace tsattn
