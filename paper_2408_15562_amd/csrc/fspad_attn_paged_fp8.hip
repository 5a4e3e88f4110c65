// Tree-masked attention over a paged 8-bit cache (arXiv 2408.15562, Preliminaries, validation phase, as fspad_attn.hip; the cache format is in
// include/fspad.h). gfx950 (CDNA4) only.
//
// The kernel of paged_attn.h on the forms of paged_forms_fp8.h. A block of 32 keys takes a wavefront of 32 rows (D = 128) 93 vector instructions and 16 products
// (540 clocks), against 155 and 16 of the 4-bit cache: the pages hold V's codes key after key, so that nothing is turned.
//
// What bounds it. Single tokens: memory. 64 sequences of 4000 tokens, 8 kv heads of D = 64 (262 MB), 49 us; 32 of them, D = 128, 50 us, 16384 tokens 188 us: 5.3 to 5.7 TB/s, 5.9 for
// longer ones. Trees on grouped heads: products and vector instructions, which do not hide each other here (64 on 8 kv heads, 60 nodes, 16384 tokens: 44 us, 750 TFLOP/s; 30 more for 16384 more,
// 1060 TFLOP/s; the same without any loads). The matrix cores are busy for 44 % of a SIMD's clocks, the vector unit for 62. Trees on heads of their own: both (4 sequences of 4096 tokens, 60 nodes and 52 heads,
// 231 MB: 59 us, 45 without loads). Of each, 6 (a token) to 11 us (trees) are starts, merges and joins.
// Tried at the last two, and not kept: exponentials and conversions between the products by scheduling groups, eight ways (60.3 to 61.0 for 60.9 us and 45.3 to 47.6 for 46.6);
// loads two turns ahead (16 rows, one token 8.8 -> 9.3 us, 32 tokens of 4000 51.1 -> 49.9; 32 rows of D = 128 spill); loads past the caches (59 -> 69 and 46 -> 58).
// How rows and keys are dealt out to wavefronts is a rule with measurements of its own, at paged_rows_fp8: 256 single tokens of 100 tokens, 32 on 8 heads 19 us and not 36; 64 trees of 60 nodes, 2000 tokens 168
// and not 249; 4 of 1000 tokens 15.7 and not 20.3.
// Units go head by head: every die then has some heads of all sequences instead of all heads of some, whose lengths differ (16 ragged trees 73.0 -> 69.6 us).
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_attn.h"
#include "paged_forms_fp8.h"
#include "paged_layout.h"
#include "paged_plan.h"

namespace {

template <int D>
void launch_rows(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  if (pl.rows_per_wave == 16) {
    if (!pl.split) launch<Form16Fp8<D>, 1, true, false>(pl, p, stream);
    else if (pl.waves == 2) launch<Form16Fp8<D>, 2, true>(pl, p, stream);
    else pl.waves == 4 ? launch<Form16Fp8<D>, 4, true>(pl, p, stream) : launch<Form16Fp8<D>, 8, true>(pl, p, stream);
  } else if (pl.rows_per_wave == 32) {
    if (!pl.split) pl.WS == 1 ? launch<Form32Fp8<D, 1>, 1, true, false>(pl, p, stream) : launch<Form32Fp8<D, 1>, 4, true, false>(pl, p, stream);
    else if (pl.waves == 2) launch<Form32Fp8<D, 1>, 2, true>(pl, p, stream);
    else pl.waves == 4 ? launch<Form32Fp8<D, 1>, 4, true>(pl, p, stream) : launch<Form32Fp8<D, 1>, 8, true>(pl, p, stream);
  } else if constexpr (D == 64) {
    pl.waves == 4 ? launch<Form32Fp8<64, 2>, 4, true>(pl, p, stream) : launch<Form32Fp8<64, 2>, 8, true>(pl, p, stream);
  }
}

}  // namespace

extern "C" size_t fspad_tree_attn_paged_byte_workspace_bytes(const fspad_paged_desc* desc) {
  if (!desc || check_paged_attn(*desc, PagedFormat::kFp8) != FSPAD_OK) return 0;
  return plan_paged(*desc, PagedFormat::kFp8).workspace_bytes;
}

extern "C" fspad_status fspad_tree_attn_paged_byte(const fspad_paged_desc* desc, const void* q, const void* k_tree, const void* v_tree,
                                                  const void* pages, const int32_t* block_table, const int32_t* kv_len,
                                                  const int32_t* n_nodes, const uint64_t* anc_mask, void* out, void* workspace,
                                                  size_t workspace_bytes, void* hip_stream) {
  return paged_attn(PagedFormat::kFp8, desc, q, k_tree, v_tree, pages, block_table, kv_len, n_nodes, anc_mask, out, workspace, workspace_bytes, hip_stream,
                    [&](const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
    desc->head_dim == 128 ? launch_rows<128>(pl, p, stream) : launch_rows<64>(pl, p, stream);
  });
}
