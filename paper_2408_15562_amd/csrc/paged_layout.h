// Where a paged 4-bit cache keeps what (include/fspad.h, "Paged 4-bit cache"). Plain host and device arithmetic, no HIP in it.
#ifndef FSPAD_PAGED_LAYOUT_H
#define FSPAD_PAGED_LAYOUT_H

#include <stdint.h>

#include "fspad.h"

namespace fspad_detail {

constexpr int kMinPageTokens = 16, kMaxPageTokens = 256;

// one kv head's part of a page: K codes, V codes, K scales, V scales
constexpr int page_code_bytes(int D, int page_tokens) { return page_tokens * D / 2; }
constexpr int page_scale_bytes(int D, int page_tokens) { return page_tokens * D / 32; }
constexpr int page_head_bytes(int D, int page_tokens) { return 2 * (page_code_bytes(D, page_tokens) + page_scale_bytes(D, page_tokens)); }

inline int log2_of(int power_of_two) { return 31 - __builtin_clz((unsigned)power_of_two); }

inline bool page_tokens_ok(int p) { return p >= kMinPageTokens && p <= kMaxPageTokens && (p & (p - 1)) == 0; }

// What every call on the pool checks of its geometry.
inline fspad_status check_pool(const fspad_paged_desc& d) {
  if (d.n_kv_heads < 1 || (d.head_dim != 64 && d.head_dim != 128) || !page_tokens_ok(d.page_tokens)) return FSPAD_ERR_SHAPE;
  if (d.io_dtype != FSPAD_BF16) return FSPAD_ERR_DTYPE;
  const int64_t page_bytes = (int64_t)d.n_kv_heads * page_head_bytes(d.head_dim, d.page_tokens);
  if (page_bytes > INT32_MAX || d.page_stride < page_bytes || d.page_stride % 16 != 0 || d.page_stride > UINT32_MAX) return FSPAD_ERR_SHAPE;
  if (d.n_pages < 1 || (int64_t)d.n_pages * d.page_tokens > INT32_MAX) return FSPAD_ERR_SHAPE;   // slots are 32-bit
  return FSPAD_OK;
}

}  // namespace fspad_detail

#endif
