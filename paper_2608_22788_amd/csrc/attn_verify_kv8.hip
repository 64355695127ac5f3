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
// What bounds it.  Long caches: bytes.  256 sequences of 500-8,000 tokens take 345 us
// (2.18 GB, 6.3 TB/s; a gather of the same 2 KiB blocks that computes nothing reaches
// 6.4-6.6), 8 sequences of 16-65 thousand with 4 rows each 107 us (5.96 TB/s).  Vector
// instructions issue in 25 % of a busy CU's cycles, the matrix units are busy 9 %.
// Two steps under way instead of one: no difference (346 against 348 us).
// One sequence of 1,600: 10 us, the chain of the launch and the join of its pieces;
// two pages per wavefront instead of four take 11.3 (more pieces).
// 33 rows and more (64 rows, 4 sequences of 32-98 thousand tokens, 146 us, 3.48 TB/s;
// 48 rows 119, 4.26): the chain of the one wavefront that a SIMD's registers hold, of
// whose time vector instructions take 36 %, matrix products 34 % and waits 25 %, one
// after the other.  17 to 32 rows (the same sequences, 32 rows, 95 us, 5.3 TB/s; memory
// alone 74) the same way: 47, 17 and 24 %.  When 64 rows took 186 us, the chunk kernel
// took 189 for them, four wavefronts that share the rows of one page 296.
// head_dim 64: 256 sequences of 500-8,000 tokens 59 us (4.9 TB/s; half of the bytes for a
// step's work), 32 of 16-65 thousand with 64 rows 137 (2.7; vector 53 %, matrix 17 %,
// waits 22 %).
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
