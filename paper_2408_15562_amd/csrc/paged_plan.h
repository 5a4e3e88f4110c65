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

// Workgroups of a compute unit. (Three of four wavefronts, D = 128, would spill: 64 sequences of 2000 tokens, 8 kv heads, 34.2 us, two 30.6.)
constexpr int paged_resident(int waves, int D, bool rows16) { return waves == 4 ? (rows16 && D == 64 ? 4 : 2) : rows16 && D == 64 ? 2 : 1; }

struct PagedPlan {
  int rows_per_wave, WS, waves;   // row slabs and wavefronts of a workgroup (those of a slab split its keys)
  int rows_per_group;    // WS * rows_per_wave: 16, 32 or 64
  int groups;            // row groups of a kv head's N * G rows
  int resident;          // workgroups that the device holds at once
  int least_blocks, whole_blocks;   // no piece is shorter, no unit of up to so many blocks is cut
  int piece_cost, join_cost, dead_cost;   // what starting and ending a piece takes, joining pieces, a unit without nodes, in blocks
  bool may_cut;          // a unit can be so long that it is cut
  bool lines;            // workgroups may take windows of all units: two slots each
  int max_pieces;
  size_t cuts_bytes, workspace_bytes;
};

inline int64_t paged_unit_blocks(const fspad_paged_desc& d) {   // at most
  return ((int64_t)d.max_kv_len + kBlockKeys - 1) / kBlockKeys + (d.n_nodes_max + kBlockKeys - 1) / kBlockKeys;
}

// Rows of a workgroup: the smallest of 16, 32 and 64 that holds all of a kv head's, or groups of 64 where none does. 64 rows are one slab with
// D = 64, two slabs of 32 with D = 128, whose wavefronts read the same keys. Four wavefronts or eight, by the rules below. A piece starts and ends
// in 8 us, pieces are joined in 5 us, and a wavefront takes 0.3 us a block when the device is full: the costs below. What is known of the lengths here
// is max_kv_len alone.
inline PagedPlan plan_paged(const fspad_paged_desc& d) {
  PagedPlan pl{};
  const int rows = d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  pl.rows_per_group = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  pl.groups = (rows + pl.rows_per_group - 1) / pl.rows_per_group;
  pl.rows_per_wave = pl.rows_per_group == 64 && d.head_dim == 128 ? 32 : pl.rows_per_group;
  pl.WS = pl.rows_per_group / pl.rows_per_wave;
  const int64_t units = (int64_t)d.batch * d.n_kv_heads * pl.groups, longest = paged_unit_blocks(d);
  // Eight wavefronts where every unit may have a compute unit to itself and they have several blocks each; else four, and workgroups that share a
  // compute unit have each other's starts and ends. One token, D = 128, 8 kv heads: 400 tokens 8.7 us on four and 9.5 on eight, 2000 13.3 and 13.2,
  // 32 sequences of 4000 32.2 and 30.7, 64 of 1000 18.2 and 21.9. 26 nodes on 32 heads: 8 sequences of 1000 15.9 and 17.5, of 2000 27.7 and 20.9, 16 of 300 .. 3000
  // 40 and 56. Two slabs (64 rows, D = 128): 60 nodes on 32 heads, 500 tokens 15.9 and 17.1, 16 sequences of 500 27.5 and 35.8, but 8 of 1000 on 8 heads of keys 33.5
  // and 24.2 (on four they are cut), 16 ragged ones of up to 6011 68 and 67: eight from 18 blocks on.
  // Few units, cut: 26 nodes on 32 heads, 2000 tokens 16.6 and 18.3, 4000 17.9 and 20.1, 8000 25.3 and 22.4; 60 nodes on 8 heads, 2000 19.2 and 21.0, on 32, 4000 27.8 and 24.3.
  // More than 32 units, on four and cut as those are, and on eight: 26 nodes on 64 heads, or 2 sequences on 32, 1300 tokens 19.9 and 16.2, 2048 20.8 and 18.9; on 40
  // heads, 1300 16.3 and 16.0, 2048 16.8 and 18.8, 3000 21.1 and 19.6.
  const bool rows16 = pl.rows_per_wave == 16;
  const bool few = !rows16 && units <= 32 && units * longest * pl.WS <= 4400;   // as many pieces of few blocks as compute units
  pl.waves = (pl.WS == 1 && units > kPagedComputeUnits) || longest <= (rows16 ? 48 : 36 / pl.WS) || few ? 4 : 8;
  const int key_waves = pl.waves / pl.WS;
  pl.resident = paged_resident(pl.waves, d.head_dim, rows16) * kPagedComputeUnits;
  pl.least_blocks = 2 * key_waves;
  // Joining costs as much as 80 blocks of 16 rows take eight wavefronts, 9 blocks a wavefront of 32 rows; cutting saves nothing where there are as
  // many units as workgroups, and half of a unit where there are half as many. One token, D = 128, 8 kv heads, whole and cut: 1 sequence of
  // 2000 tokens 13.2 and 13.5 us, 4000 18.1 and 14.9, 8000 27.5 and 16.5; 16 sequences of 4000 18.8 and 20.2, 8000 35.9 and 35.1; 32 of
  // 8000 53.7 and 56.1; 64 of 250 .. 4000, D = 64, 20.3 and 25.2. 26 nodes on 32 heads, eight wavefronts: 2048 19.6 and 19.4; 3000 22.8 and 19.8.
  const int cuts = (int)(kPagedComputeUnits / units);
  pl.whole_blocks = !rows16 ? 9 * key_waves : pl.waves == 4 ? 128 : cuts < 2 ? 256 : 80 * cuts / (cuts - 1);
  pl.piece_cost = 8 * key_waves;
  pl.join_cost = 4 * key_waves;
  pl.dead_cost = key_waves;
  pl.may_cut = d.workgroups > 0 || longest > pl.whole_blocks;
  // as many as there may be blocks, but at most two rounds of the device beside one for each unit
  int64_t cut = d.workgroups > 0 ? d.workgroups : 2 * pl.resident;
  if (cut > units * longest) cut = units * longest;
  pl.max_pieces = (int)(units + (pl.may_cut ? cut : 0));
  pl.lines = pl.rows_per_wave > 16 && pl.max_pieces >= 2 * pl.resident;
  pl.cuts_bytes = (size_t)((units * 8 + 15) / 16 * 16);
  pl.workspace_bytes = pl.cuts_bytes + (pl.may_cut ? (size_t)pl.max_pieces * pl.rows_per_group * (d.head_dim + 2) * 4 : 0);
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
  // 32-bit rows, units and blocks of all units, and launch dimensions
  const int64_t rows = (int64_t)d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  if (rows > (1 << 20) || d.n_kv_heads > 65535) return FSPAD_ERR_SHAPE;
  const PagedPlan pl = plan_paged(d);
  if ((int64_t)d.batch * pl.groups > 65535) return FSPAD_ERR_SHAPE;
  if ((int64_t)d.batch * d.n_kv_heads * pl.groups * paged_unit_blocks(d) > (1 << 30)) return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

}  // namespace fspad_detail

#endif
