// Running sum and maximum over a wavefront's lanes, internal to the library. gfx950 (CDNA4) only.
#ifndef FSPAD_WAVE_SCAN_H
#define FSPAD_WAVE_SCAN_H

#include <hip/hip_runtime.h>

namespace fspad_detail {

// Sum of x over the lanes up to and including this one: within rows of 16 lanes by shifts, then the rows' last lanes to the rows
// behind them. No trip through LDS.
__device__ __forceinline__ int wave_sum_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // row_shr 1, 2, 4, 8 (zeros come in)
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
  return x;
}

// The largest of x >= 0 over the lanes up to and including this one.
__device__ __forceinline__ int wave_max_upto(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return x;
}

}  // namespace fspad_detail

#endif
