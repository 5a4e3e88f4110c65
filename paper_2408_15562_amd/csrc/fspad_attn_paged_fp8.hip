// Tree-masked attention over a paged 8-bit cache (arXiv 2408.15562, Preliminaries, validation phase, as fspad_attn.hip; the cache format is in
// include/fspad.h). gfx950 (CDNA4) only.
//
// The kernel of paged_attn.h on the forms of paged_forms_fp8.h.
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
  if (pl.rows_per_wave == 16) pl.waves == 4 ? launch<Form16Fp8<D>, 4, true>(pl, p, stream) : launch<Form16Fp8<D>, 8, true>(pl, p, stream);
  else if (pl.rows_per_wave == 32) pl.waves == 4 ? launch<Form32Fp8<D, 1>, 4, true>(pl, p, stream) : launch<Form32Fp8<D, 1>, 8, true>(pl, p, stream);
  else if constexpr (D == 64) pl.waves == 4 ? launch<Form32Fp8<64, 2>, 4, true>(pl, p, stream) : launch<Form32Fp8<64, 2>, 8, true>(pl, p, stream);
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
