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
// Slabs of their own, four of them, D = 64: three, although 31 registers go to memory: 64 trees of 60 nodes on 32 heads, 8 of keys, 500 tokens 43 -> 39 us, 2000 tokens 113 -> 100; one slab of 32 rows
// would lose by it (256 of 7 nodes, 250 tokens 21.0 -> 22.4).
constexpr int paged_resident(int waves, int D, bool rows16, bool split) { return (D == 128 ? 8 : rows16 ? 16 : !split && waves == 4 ? 12 : 8) / waves; }

constexpr int kSlabWhole = 96;   // units of so many blocks are not cut where a slab has four wavefronts or fewer, 8-bit

struct PagedPlan {
  int rows_per_wave, WS, waves;   // row slabs and wavefronts of a workgroup (those of a slab split its keys)
  int rows_per_group;    // WS * rows_per_wave: 16, 32, 64 or 128
  int groups;            // row groups of a kv head's N * G rows
  int resident;          // workgroups that the device holds at once
  int least_blocks, whole_blocks;   // no piece is shorter, no unit of up to so many blocks is cut
  int piece_cost, join_cost, dead_cost;   // what starting and ending a piece takes, joining pieces, a unit without nodes, in blocks
  bool split;            // a slab's wavefronts split its keys, else there is one
  bool may_cut;          // a unit can be so long that it is cut
  bool lines;            // workgroups may take windows of all units: two slots each
  int max_pieces;
  size_t cuts_bytes, workspace_bytes;
};

inline int64_t paged_unit_blocks(const fspad_paged_desc& d) {   // at most
  return ((int64_t)d.max_kv_len + kBlockKeys - 1) / kBlockKeys + (d.n_nodes_max + kBlockKeys - 1) / kBlockKeys;
}

// How a call over the 8-bit cache deals its rows out: in slabs of 16 or 32 rows (WS of them a workgroup), and a slab's keys to `key_waves` wavefronts.
// Two slabs, or one of 64 rows, in a workgroup read keys once for both (the 4-bit cache's way); a workgroup of one slab is lighter, and a wavefront that
// has all keys of its rows merges nothing. Below, us: by the rule / the 4-bit way, or slabs x wavefronts of a slab; D = 128 where nothing is said,
// query heads on kv heads. profiles/paged_fp8_dealing.txt has every way for 48 calls, and 200 drawn calls by the rule and the 4-bit way.
//  - No more slabs than compute units: one a workgroup, four wavefronts up to 72 blocks, then eight if the pieces fill three quarters of the device.
//    4 x 60 nodes, 16 on 16: 300 tokens 10.5 / 13.1, 1 x 8 12.3; 2000 17.3 / 22.4, 1 x 8 18.0. 32 on 8: 2000 17.5 / 26.8; 4000 25.7 / 31.7, 1 x 4 31.6.
//    D = 64: 1000 10.6 / 15.2, 1 x 8 11.0; 4000 17.1 / 25.3, 1 x 4 22.8. 1 x 60 nodes, 64 on 8, 16384: 44.0 / 44.9
//  - More: the same on four wavefronts up to 72 blocks, D = 128 from 37 on. 4 x 60 nodes, 64 on 8: 2000 26.0 / 28.6; D = 64 500 12.0 / 13.4, 2000 18.3 / 20.7;
//    as the 4-bit cache: 500 15.3, 1 x 4 16.1; 36 nodes, 40 on 40, 8000 82, 1 x 4 111, 1 x 2 76
//  - Three a compute unit (16 rows: four; long ones, D = 64: six) and more than 64 rows: four a workgroup, a wavefront each. 60 nodes, 32 on 8: 12 sequences of
//    50 .. 4000 53 / 58, 1 x 4 60; 64 of 500 64 / 83, 1 x 4 110; 64 of 2000 166 / 245. D = 64: 64 of 500 38 / 66, 1 x 4 78. It loses a little where a unit is long
//    and the device has no more than two rounds of them: D = 64, 12 of 2000 30.0 / 31.9, 1 x 4 25.3; 101 of 39 nodes, 48 on 12, 7250 769 / 665
//  - The same, 64 rows or fewer, up to 72 blocks: a slab a workgroup, one wavefront where they are short or six a compute unit, else two. One token, 32 on 8:
//    128 of 30 8.1 / 11.9, 256 of 100 17.8 / 34.1, 1 x 2 23.4, 128 of 500 25.0 / 28.0, 1 x 1 26.8. 7 nodes: 96 of 500 24.1 / 26.8, 1 x 1 23.7, 256 of 500 53 / 70, 1 x 2 58;
//    D = 64, 96 of 50 .. 2000 27.7 / 34.9, 1 x 1 30.2. 60 nodes, 16 on 16: 32 of 1000 31.7 / 40.6
//  - More than 32 rows and few keys: one wavefront a slab. 60 nodes, 32 on 8: one token 9.8 / 11.0, 150 11.5 / 12.3; D = 64: 8.1 / 9.0, 250 10.6 / 11.5 (1 x 4, which was
//    measured after the rule was made: 8.4, 9.8, 6.7, 8.4)
struct PagedRows {
  int per_wave, WS, key_waves;   // key_waves 0: as over the 4-bit cache
};
inline PagedRows paged_rows_fp8(const fspad_paged_desc& d, int rows, int64_t longest) {
  const int per_wave = rows <= 16 ? 16 : 32;
  const int64_t slabs = (int64_t)d.batch * d.n_kv_heads * ((rows + per_wave - 1) / per_wave);
  const bool many = slabs >= (rows <= 16 ? 4 : d.head_dim == 64 && longest > kSlabWhole ? 6 : 3) * kPagedComputeUnits;
  if (many && rows > 64) return {per_wave, 4, 1};
  if (rows > 32 && longest <= (d.head_dim == 64 ? 10 : 7)) return {per_wave, 1, 1};
  if (many && longest <= 72) return {per_wave, 1, longest <= (rows <= 16 ? 8 : 12) || slabs >= 6 * kPagedComputeUnits ? 1 : 2};
  if (rows <= 16) return {16, 1, 0};
  if (slabs <= kPagedComputeUnits) {
    if (longest <= 72) return {32, 1, 4};
    if (rows <= 32 || kPagedComputeUnits / slabs * slabs >= 192) return {32, 1, 8};
  }
  if (rows <= 32 || (longest <= 72 && (d.head_dim == 64 || longest > 36))) return {32, 1, 4};
  return {32, 1, 0};
}

// Rows of a workgroup: the smallest of 16, 32 and 64 that holds all of a kv head's, or groups of 64 where none does. 64 rows are one slab with
// D = 64, two slabs of 32 with D = 128, whose wavefronts read the same keys; over the 8-bit cache by the rule above, where it gives one. Four wavefronts or eight, by the rules below. A piece starts and ends
// in 8 us, pieces are joined in 5 us, and a wavefront takes 0.3 us a block when the device is full: the costs below. What is known of the lengths here
// is max_kv_len alone.
inline PagedPlan plan_paged(const fspad_paged_desc& d, PagedFormat format = PagedFormat::kFp4) {
  PagedPlan pl{};
  const int rows = d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  pl.rows_per_group = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  pl.groups = (rows + pl.rows_per_group - 1) / pl.rows_per_group;
  pl.rows_per_wave = pl.rows_per_group == 64 && d.head_dim == 128 ? 32 : pl.rows_per_group;
  pl.WS = pl.rows_per_group / pl.rows_per_wave;
  const int64_t longest = paged_unit_blocks(d);
  const PagedRows dealt = format == PagedFormat::kFp8 ? paged_rows_fp8(d, rows, longest) : PagedRows{};
  if (dealt.key_waves) {
    pl.rows_per_wave = dealt.per_wave;
    pl.WS = dealt.WS;
    pl.rows_per_group = pl.WS * pl.rows_per_wave;
    pl.groups = (rows + pl.rows_per_group - 1) / pl.rows_per_group;
  }
  pl.split = dealt.key_waves != 1;
  const int64_t units = (int64_t)d.batch * d.n_kv_heads * pl.groups;
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
  pl.waves = dealt.key_waves ? dealt.key_waves * pl.WS : (pl.WS == 1 && units > kPagedComputeUnits) || longest <= (rows16 ? 48 : 36 / pl.WS) || few ? 4 : 8;
  const int key_waves = pl.waves / pl.WS;
  pl.resident = paged_resident(pl.waves, d.head_dim, rows16, pl.split) * kPagedComputeUnits;
  pl.least_blocks = 2 * key_waves;
  // Joining costs as much as 80 blocks of 16 rows take eight wavefronts, 9 blocks a wavefront of 32 rows; cutting saves nothing where there are as
  // many units as workgroups, and half of a unit where there are half as many. One token, D = 128, 8 kv heads, whole and cut: 1 sequence of
  // 2000 tokens 13.2 and 13.5 us, 4000 18.1 and 14.9, 8000 27.5 and 16.5; 16 sequences of 4000 18.8 and 20.2, 8000 35.9 and 35.1; 32 of
  // 8000 53.7 and 56.1; 64 of 250 .. 4000, D = 64, 20.3 and 25.2. 26 nodes on 32 heads, eight wavefronts: 2048 19.6 and 19.4; 3000 22.8 and 19.8.
  const int cuts = (int)(kPagedComputeUnits / units);
  pl.whole_blocks = !rows16 ? 9 * key_waves : pl.waves == 4 ? 128 : cuts < 2 ? 256 : 80 * cuts / (cuts - 1);
  // 8-bit: 8 sequences of 1000 tokens, 60 nodes on 64 heads, 8 of keys, on one wavefront 41 us cut, 29 whole; 16 on 32 heads of 2000 59 and 45; 32 of 100 .. 4000 94 and 106. On four, 4 of 2000 on 32 heads 29 and 20.
  if (dealt.key_waves) pl.whole_blocks = key_waves <= 4 ? kSlabWhole : cuts < 2 ? 256 : 80 * cuts / (cuts - 1);
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

inline fspad_status check_paged_attn(const fspad_paged_desc& d, PagedFormat format = PagedFormat::kFp4) {
  if (const fspad_status st = check_pool(d, format)) return st;
  if (d.batch < 1 || d.batch > kPagedMaxBatch || d.n_nodes_max < 1 || d.n_nodes_max > FSPAD_MAX_NODES) return FSPAD_ERR_SHAPE;
  if (d.n_q_heads < 1 || d.n_q_heads % d.n_kv_heads != 0) return FSPAD_ERR_SHAPE;
  if (d.out_dtype != FSPAD_BF16 && d.out_dtype != FSPAD_F32) return FSPAD_ERR_DTYPE;
  if (d.table_width < 1 || d.table_stride < d.table_width || (int64_t)d.table_width * d.page_tokens > INT32_MAX) return FSPAD_ERR_SHAPE;
  if (d.max_kv_len < 0 || d.max_kv_len > d.table_width * d.page_tokens) return FSPAD_ERR_SHAPE;
  if (d.workgroups < 0 || d.workgroups > 4096) return FSPAD_ERR_SHAPE;
  // 32-bit rows, units and blocks of all units, and launch dimensions
  const int64_t rows = (int64_t)d.n_nodes_max * (d.n_q_heads / d.n_kv_heads);
  if (rows > (1 << 20) || d.n_kv_heads > 65535) return FSPAD_ERR_SHAPE;
  const PagedPlan pl = plan_paged(d, format);
  if ((int64_t)d.batch * pl.groups > 65535) return FSPAD_ERR_SHAPE;
  if ((int64_t)d.batch * d.n_kv_heads * pl.groups * paged_unit_blocks(d) > (1 << 30)) return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

}  // namespace fspad_detail

#endif
