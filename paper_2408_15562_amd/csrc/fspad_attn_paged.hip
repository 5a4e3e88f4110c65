// Tree-masked attention over a paged 4-bit cache (arXiv 2408.15562, Preliminaries, validation phase, as fspad_attn.hip; the
// cache format is in include/fspad.h). gfx950 (CDNA4) only.
//
// One pass over the keys with a running shift and sum per query row. A wavefront owns 16, 32 or 64 query rows of one kv head and takes 32-key
// blocks of K and V from the pages straight into registers, 4 bits an entry; the layout of the pages is that of the operands:
//   S^T = K Q^T    on the block-scaled products, which take K's codes and scales as they are. They have no bf16 operand; a query row
//                  is two fp8 ones instead (split_row), whose sum it is. As many clocks as bf16 products take, and nothing to convert.
//   O^T += V^T P^T V's scales run along the channels, not along the keys that are summed over, so V becomes bf16
//                  (v_cvt_scalef32_pk_bf16_fp4: two entries and their block's scale in one instruction, exact), and turns from key
//                  order to channel order two bytes at a time (v_perm_b32).
// paged_forms.h has both, for 16 rows and for tiles of 32.
//
// What bounds it: instructions. A block of 32 keys takes a wavefront of 32 rows (D = 128) 155 vector instructions, 92 of them V's, and
// 540 clocks of products, and of the two wavefronts of a SIMD the products of one hide little of the other's vector work: 1060 clocks a
// block for one wavefront alone, 960 for each of two (probed without loads; 1120 and 990 with them). 64 query heads on 8 kv heads, 60 nodes, 16384 tokens
// (32 GFLOP): 48 us, 5 of them the join's, 670 TFLOP/s; 4 sequences of 4096 tokens, 60 nodes and 52 heads (116 MB of pages, 129 with the rows): 49 us, 4 of
// them a join without pieces, 2.6 TB/s.
// Both sides of what was chosen, at these two, the kernel alone under a profiler: 64 rows a wavefront (D = 128, one wavefront a SIMD, V converted once for all)
// 55 and 55 us for 51 and 51; with D = 64 64 rows fit two wavefronts a SIMD and win, 33 for 34.5 us (8 sequences of 4000) and 68 for 72 us (32 ragged ones).
//
// How a call is cut is decided on the device, from lengths it alone knows (piece_length): a unit, 64 query rows or less of one kv head of one
// sequence, is one workgroup's or is cut along its keys. A whole unit goes straight to `out`; of the others every piece leaves its
// un-normalised sums in the workspace and a second kernel joins them.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_attn.h"
#include "paged_forms.h"
#include "paged_layout.h"
#include "paged_plan.h"

namespace {

template <int D, bool WIDE>
void launch_rows(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  if (pl.rows_per_wave == 16) pl.waves == 4 ? launch<Form16<D>, 4, WIDE>(pl, p, stream) : launch<Form16<D>, 8, WIDE>(pl, p, stream);
  else if (pl.rows_per_wave == 32) pl.waves == 4 ? launch<Form32<D, 1>, 4, WIDE>(pl, p, stream) : launch<Form32<D, 1>, 8, WIDE>(pl, p, stream);
  else if constexpr (D == 64) pl.waves == 4 ? launch<Form32<64, 2>, 4, WIDE>(pl, p, stream) : launch<Form32<64, 2>, 8, WIDE>(pl, p, stream);
}

}  // namespace


extern "C" size_t fspad_tree_attn_paged_workspace_bytes(const fspad_paged_desc* desc) {
  if (!desc || check_paged_attn(*desc, PagedFormat::kFp4) != FSPAD_OK) return 0;
  return plan_paged(*desc, PagedFormat::kFp4).workspace_bytes;
}

extern "C" fspad_status fspad_tree_attn_paged(const fspad_paged_desc* desc, const void* q, const void* k_tree, const void* v_tree,
                                              const void* pages, const int32_t* block_table, const int32_t* kv_len,
                                              const int32_t* n_nodes, const uint64_t* anc_mask, void* out, void* workspace,
                                              size_t workspace_bytes, void* hip_stream) {
  return paged_attn(PagedFormat::kFp4, desc, q, k_tree, v_tree, pages, block_table, kv_len, n_nodes, anc_mask, out, workspace, workspace_bytes, hip_stream,
                    [&](const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
    const bool wide = desc->page_tokens >= kBlockKeys;
    if (desc->head_dim == 128) wide ? launch_rows<128, true>(pl, p, stream) : launch_rows<128, false>(pl, p, stream);
    else wide ? launch_rows<64, true>(pl, p, stream) : launch_rows<64, false>(pl, p, stream);
  });
}
