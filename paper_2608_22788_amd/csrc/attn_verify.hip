// attn_verify.hip -- paged speculative-verify attention: each sequence
// brings q_len = 1 + gamma query rows (the draft block) that attend to the
// whole cache and causally to each other, on bf16 matrix cores.
//
// The G query heads of a KV group times the q_len draft rows form
// R = G * Qmax rows per (sequence, KV head) unit, padded to NB blocks of 16;
// row r is draft position i = r / G of query head g * G + r % G.  One
// wavefront streams the unit's pages and keeps every row block in registers,
// so each K/V byte is read once for all rows of the group.
//
// With l = lane, n = l % 16, kq = l / 16, per 16-token page:
//   * scores S^T = K Q^T on v_mfma_f32_16x16x32_bf16 (A: row l%16, k
//     8(l/16)..+7; B: col l%16, k 8(l/16)..+7; C: row 4(l/16)+i, col l%16):
//     A = 16 key rows x 32 dims loaded straight from the page (16 bytes per
//     lane), B = Q^T kept in registers.  Lane (n, kq) receives tokens
//     4kq..4kq+3 of the page for query row n;
//   * probabilities P = exp2(scale*log2e * S - m_ref), packed to bf16 in the
//     lane that computed them, are exactly the A operand of O = P V on
//     v_mfma_f32_16x16x16_bf16 (A: row l%16, k 4(l/16)..+3);
//   * V is loaded as rows (lane (n, kq) reads D/16 consecutive dims of tokens
//     4kq..4kq+3) and transposed in registers, so the B operand of the j-th
//     P.V product holds dims (D/16) n + j of those four tokens;
//   * row sums come from one more product of P with a ones operand, so they
//     use exactly the rounded probabilities that weight V;
//   * the running reference m_ref of each row is only raised when a score
//     exceeds it by more than 8 in log2 units, which leaves the accumulators
//     untouched on almost every page;
//   * the next page is loaded into a second register set while the current
//     one is computed; loads go through a buffer resource bounded to the
//     page's block, so a prefetch past the end reads nothing (it used to
//     re-read the last page: about 0.8 % of the bulk call's traffic).  With
//     one row block the prefetch runs on across the end of a segment into
//     the next segment's first page, whose lengths and query rows are
//     fetched when the current segment starts, so the pipeline is not
//     drained at a unit boundary.
// Masks: key t is visible to draft row i iff t <= L - Q + i; keys past the
// segment end or the context end get probability 0 and their value rows are
// zeroed before the product, so stale data never reaches the output.
// Splits are combined as p.combine says (attn_split.h): by the last worker to
// finish a piece of the unit, by the merge wavefronts that follow the workers
// in the grid (workgroups W and up), or by the separate merge kernel.
//
// Two kernels share this code: verify_kernel, where a wavefront is a worker,
// and verify_group_kernel (the automatic choice), where four are and the
// pieces of a unit that they share meet in LDS first.
#include "attn_verify.h"

namespace tsattn {

typedef void (*kernel_fn)(AttnParams);

// The group kernel and its LDS need beyond the prefix.
kernel_fn verify_group_variant(int D, int NB, int *lds_bytes) {
#define TS_VG(DD, NN)                                                \
    if (D == DD && NB == NN) {                                       \
        *lds_bytes = (int)sizeof(typename Verify<DD, NN, false>::GroupLds); \
        return verify_group_kernel<DD, NN, false>;                          \
    }
    TS_VG(64, 1) TS_VG(64, 2) TS_VG(64, 3) TS_VG(64, 4) TS_VG(128, 1) TS_VG(128, 2)
#undef TS_VG
    return nullptr;
}

kernel_fn verify_variant(int D, int NB) {
#define TS_VF(DD, NN) \
    if (D == DD && NB == NN) return verify_kernel<DD, NN, false>;
    TS_VF(64, 1) TS_VF(64, 2) TS_VF(64, 3) TS_VF(64, 4)
    TS_VF(128, 1) TS_VF(128, 2) TS_VF(128, 3) TS_VF(128, 4)
#undef TS_VF
    return nullptr;
}

}  // namespace tsattn
