// How a call of the attention over a paged cache is laid out: rows per workgroup, number of workgroups, workspace. Plain host
// code, no HIP in it.
#ifndef FSPAD_PAGED_PLAN_H
#define FSPAD_PAGED_PLAN_H

#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"

namespace fspad_detail {

constexpr int kBlockKeys = 32;
constexpr int kPagedMaxBatch = 1024;
constexpr int kPagedComputeUnits = 256;

struct PagedPlan {
  int QT, WS;            // 16-row tiles of a wavefront, row slabs of a workgroup (4 / WS wavefronts split a slab's keys)
  int rows_per_group;    // WS * 16 * QT
  int groups;            // row groups of a kv head's N * G rows
  int n_wgs, min_blocks; // workgroups at most; blocks that a workgroup is worth
  size_t cuts_bytes, workspace_bytes;
};

inline int64_t paged_places(const fspad_paged_desc& d, int groups) {   // of the list, at most
  const int64_t blocks = ((int64_t)d.max_kv_len + kBlockKeys - 1) / kBlockKeys + (d.n_nodes_max + kBlockKeys - 1) / kBlockKeys;
  return (int64_t)d.batch * d.n_kv_heads * groups * blocks;
}

// Up to 64 rows: one slab, the four wavefronts split the keys. Up to 128: two slabs; more: four, in groups of up to 256 rows.
inline PagedPlan plan_paged(const fspad_paged_desc& d) {
  PagedPlan pl{};
  const int rows = d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  pl.groups = (rows + 255) / 256;
  const int share = (rows + pl.groups - 1) / pl.groups;
  pl.WS = share <= 64 ? 1 : share <= 128 ? 2 : 4;
  pl.QT = (share + 16 * pl.WS - 1) / (16 * pl.WS);
  pl.rows_per_group = pl.WS * 16 * pl.QT;
  pl.min_blocks = 2 * (4 / pl.WS);
  const int64_t places = paged_places(d, pl.groups);
  int64_t wgs = pl.QT <= 2 ? 2 * kPagedComputeUnits : kPagedComputeUnits;
  if (d.workgroups > 0) {
    wgs = d.workgroups;
    pl.min_blocks = 1;
  }
  const int64_t most = places / pl.min_blocks > 1 ? places / pl.min_blocks : 1;
  pl.n_wgs = (int)(wgs < most ? wgs : most);
  const int64_t units = (int64_t)d.batch * d.n_kv_heads * pl.groups;
  pl.cuts_bytes = (size_t)((units * 8 + 15) / 16 * 16);
  pl.workspace_bytes = pl.cuts_bytes + (size_t)(units + pl.n_wgs) * pl.rows_per_group * (d.head_dim + 2) * 4;
  return pl;
}

inline fspad_status check_paged_attn(const fspad_paged_desc& d) {
  if (const fspad_status st = check_pool(d)) return st;
  if (d.batch < 1 || d.batch > kPagedMaxBatch || d.n_nodes_max < 1 || d.n_nodes_max > FSPAD_MAX_NODES) return FSPAD_ERR_SHAPE;
  if (d.n_q_heads < 1 || d.n_q_heads % d.n_kv_heads != 0) return FSPAD_ERR_SHAPE;
  if (d.out_dtype != FSPAD_BF16 && d.out_dtype != FSPAD_F32) return FSPAD_ERR_DTYPE;
  if (d.table_width < 1 || d.table_stride < d.table_width || (int64_t)d.table_width * d.page_tokens > INT32_MAX) return FSPAD_ERR_SHAPE;
  if (d.max_kv_len < 0 || d.max_kv_len > d.table_width * d.page_tokens) return FSPAD_ERR_SHAPE;
  if (d.workgroups < 0 || d.workgroups > 4096) return FSPAD_ERR_SHAPE;
  // 32-bit places, units and launch dimensions
  const int64_t rows = (int64_t)d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  const int64_t groups = (rows + 255) / 256;
  if (rows > (1 << 20) || d.n_kv_heads * groups > 65535) return FSPAD_ERR_SHAPE;
  if (paged_places(d, (int)groups) > (1 << 30)) return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

}  // namespace fspad_detail

#endif
