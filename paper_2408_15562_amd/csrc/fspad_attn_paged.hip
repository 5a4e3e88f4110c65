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
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "fspad.h"
#include "paged_forms.h"
#include "paged_layout.h"
#include "paged_plan.h"
#include "stream_gemm.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// What is known of how a call is cut before its lengths are.
struct CutArgs {
  const int32_t* kv_len;
  const int32_t* n_nodes;
  int32_t B, N, G, Hkv, rows_shift, ws_shift, groups, max_kv_len, resident, max_pieces, least_blocks, whole_blocks, piece_cost, join_cost, dead_cost, lines, uncut, forced;   // uncut: every unit is one piece
};

struct PagedParams {
  CutArgs cut;
  const char* q;
  const char* k_tree;
  const char* v_tree;
  const char* pages;
  const int32_t* table;
  const uint64_t* mask;
  void* out;
  int2* cuts;       // per unit: first partial slot and number of pieces (0: the unit is complete in `out`; negative: of windows)
  float* part;      // partial slots, one for every piece
  int64_t table_stride;
  uint32_t page_stride;
  int32_t B, N, Hq, Hkv, G, page_shift, n_pages;
  uint32_t g_rcp;   // reciprocal(G)
  int32_t ws_shift, rows_per_group, groups, out_bf16;
  float c;          // softmax scale * log2(e)
};

// The arguments where the launch left them. What only a segment's start or end needs is fetched there, through a pointer that the
// compiler takes for another one each time: kept in scalar registers for the length of a stream, arguments displaced what the stream needs.
typedef const __attribute__((address_space(4))) PagedParams* Args;
__device__ __forceinline__ Args fresh(Args p) {
  asm volatile("" : "+s"(p));
  return p;
}
// All at once: fetched where each is used, they would be waited for one after the other.
__device__ __forceinline__ CutArgs cut_args(Args p) {
  p = fresh(p);
  CutArgs a{p->cut.kv_len, p->cut.n_nodes, p->cut.B, p->cut.N, p->cut.G, p->cut.Hkv, p->cut.rows_shift, p->cut.ws_shift, p->cut.groups,
            p->cut.max_kv_len, p->cut.resident, p->cut.max_pieces, p->cut.least_blocks, p->cut.whole_blocks, p->cut.piece_cost, p->cut.join_cost, p->cut.dead_cost, p->cut.lines, p->cut.uncut, p->cut.forced};
  asm volatile("" : "+s"(a.kv_len), "+s"(a.n_nodes), "+s"(a.B), "+s"(a.N), "+s"(a.G), "+s"(a.Hkv), "+s"(a.rows_shift), "+s"(a.ws_shift), "+s"(a.groups));
  asm volatile("" : "+s"(a.max_kv_len), "+s"(a.resident), "+s"(a.max_pieces), "+s"(a.least_blocks), "+s"(a.whole_blocks), "+s"(a.piece_cost),
                    "+s"(a.join_cost), "+s"(a.dead_cost), "+s"(a.lines), "+s"(a.uncut), "+s"(a.forced));
  return a;
}

// The shift of a row moves only when a score exceeds it by more than this (log2 units): weights stay below 2^8, which fp32 sums
// and bf16 weights hold without loss, and accumulators are rescaled almost never after the first blocks.
constexpr float kLazyLog2 = 8.0f;
constexpr float kNoShift = -FLT_MAX;   // below every score: the first visible one moves it

// ------------------------------------------------------------------------------------------------ plan

// What a sequence is made of: `live` row groups of nb blocks each per kv head, the others without nodes (they write zeros). Where the last
// of them has rows for one slab of two only, all wavefronts share that slab's keys: two of its blocks take as long as one of another.
struct SeqShape {
  int len, n, live, nb, half;   // half: 1 for such a last group, else 0
};
__device__ __forceinline__ int2 seq_at(const CutArgs& p, int b) { return b < p.B ? make_int2(p.kv_len[b], p.n_nodes[b]) : make_int2(0, 0); }
template <bool SLABS>
__device__ __forceinline__ SeqShape shape_of(const CutArgs& p, int2 seq) {
  SeqShape s;
  s.len = min(max(seq.x, 0), p.max_kv_len);
  s.n = min(max(seq.y, 0), p.N);
  s.live = (s.n * p.G + (1 << p.rows_shift) - 1) >> p.rows_shift;
  s.nb = s.live > 0 ? (s.len + kBlockKeys - 1) / kBlockKeys + (s.n + kBlockKeys - 1) / kBlockKeys : 0;
  s.half = SLABS && p.ws_shift > 0 && 2 * (s.n * p.G - (s.live - 1) * (1 << p.rows_shift)) <= (1 << p.rows_shift) ? 1 : 0;
  return s;
}

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

// How a call is cut. More than 0: units are cut into equal pieces of so many blocks at most, as many as the device holds workgroups
// at once where that can be (they take as long as the longest of them). 0: all units one behind the other make a line, and every
// workgroup takes an equal window of it: the end of one unit, whole ones, the start of another. What starting and ending a piece takes
// stands on the line as blocks in front of each unit. 16 ragged sequences of 131 .. 6011 tokens, 17 .. 60 nodes on 32 heads (8 of keys): 99 us in
// equal pieces or whole units, several a workgroup, 69 us on a line; 32 of 100 .. 4000 tokens, D = 64: 96 and 68 us. Where all units go in
// one round the line costs a second start for most workgroups: 53 for 49 us (64 units, 256 workgroups). With 16 rows, D = 64, two or four
// workgroups share a compute unit and each other's gaps: 64 ragged sequences of one token 27 us on a line, 25 us in equal pieces (whole, as they
// are now, 19); 16 rows never go on a line.
template <bool LINES>
__device__ __forceinline__ int piece_length(const CutArgs& p, int blocks, int units, int longest) {
  const float slots = (float)(p.max_pieces - p.B * p.Hkv * p.groups);   // the sum of ceil(nb / len) is at most S / len + units
  if (p.forced > 0) return max((int)ceilf((float)blocks / slots) + 1, 1);
  if (longest <= p.whole_blocks) return max(longest, 1);
  const float R = (float)p.resident, S = (float)blocks, U = (float)units, cost = (float)p.piece_cost, join = (float)p.join_cost;
  // A unit of n pieces takes its longest piece and n / 8 trips to memory in the join, 0.1 us a block and about 1.6 us: pieces of the
  // root of (its blocks times half the wavefronts that share them) at least. One token, 8 kv heads: 16384 tokens 37 us in pieces of 8 blocks, 20 us; 40000 48 and 25 us.
  const float least = fmaxf((float)p.least_blocks, ceilf(__builtin_sqrtf(0.25f * (float)p.least_blocks * (float)longest)));
  float len = (float)longest, time = len + cost;
  if (units <= p.resident) {
    const float one = fminf(U < R ? ceilf(S / (R - U)) : len, ceilf(len / floorf(R / U)));   // either way there are at most R pieces
    if (one < len) {
      len = one;
      time = one + cost + join;
    }
  }
  const int equal = (int)fmaxf(fmaxf(len, least), ceilf(S / slots) + 1.0f);
  if constexpr (!LINES) return equal;
  const float line = S + U * cost + (float)p.dead_cost * (float)(p.B * p.Hkv * p.groups);
  if (p.lines && line < 1e9f && (units > p.resident || line / R + 1.5f * cost + join < time)) return 0;
  return equal;
}

// The pieces of this workgroup. Units are numbered sequence by sequence, head by head, group by group, and behind a sequence's others those
// without nodes; workgroups eight apart, which share a die and its L2 cache, take neighbouring pieces or windows.
struct Piece {
  int b, g, y, len, n, half, begin, end, index, count;   // blocks [begin, end) of a unit; index: its slot; count: pieces of the unit
  bool dead;
};
// LINES: windows may be what the call is cut into; SLABS: workgroups have two of them, or one.
template <bool LINES, bool SLABS>
struct Cutter {
  int lane, most, window, length;   // length: of the line of units, in pieces or in blocks
  int2 seq;                 // 64 sequences at a time, one a lane, from `first` on: length and nodes
  int first, before, in_these;   // the line's length before theirs, and theirs
  int at, stop, step;       // this workgroup's next place on the line; the end and the step of them

  struct Counts {
    SeqShape s;
    int unit, head, own, upto;   // lengths on the line: of a unit, of a head's, of the sequence, of the sequences up to it
  };
  __device__ __forceinline__ bool by_pieces() const { return !LINES || most > 0; }
  __device__ __forceinline__ int dead_length(const CutArgs& p) const { return by_pieces() ? 1 : p.dead_cost; }
  __device__ __forceinline__ Counts count(const CutArgs& p) const {
    Counts c;
    c.s = shape_of<SLABS>(p, seq);
    const int blocks = (c.s.nb + c.s.half) >> c.s.half;   // of the last group, as long as others' take
    c.unit = p.uncut ? 1 : by_pieces() ? (c.s.nb + most - 1) / most : c.s.nb + p.piece_cost;
    int tail = c.unit;
    if (SLABS && c.s.half && !p.uncut) tail = by_pieces() ? (blocks + most - 1) / most : blocks + p.piece_cost;
    c.head = c.s.live == 0 ? 0 : (c.s.live - 1) * c.unit + tail;
    c.own = first + lane < p.B ? p.Hkv * (c.head + (p.groups - c.s.live) * dead_length(p)) : 0;
    c.upto = wave_sum_upto(c.own);
    return c;
  }
  __device__ __forceinline__ Cutter(const CutArgs& p, int lane_) : lane(lane_) {
    seq = seq_at(p, lane);
    most = 1;
    if (!p.uncut) {
      int blocks = 0, units = 0, longest = 0;
      for (first = 0;;) {
        const SeqShape s = shape_of<SLABS>(p, seq);
        blocks += last_lane(wave_sum_upto(p.Hkv * (s.live * s.nb - (s.half ? s.nb / 2 : 0))));
        units += last_lane(wave_sum_upto(p.Hkv * s.live));
        longest = max(longest, last_lane(wave_max_upto(s.nb)));
        first += 64;
        if (first >= p.B) break;
        seq = seq_at(p, first + lane);
      }
      most = __builtin_amdgcn_readfirstlane(piece_length<LINES>(p, blocks, units, longest));
    }
    length = 0;
    for (first = 0;; first += 64) {
      if (p.B > 64) seq = seq_at(p, first + lane);
      in_these = last_lane(count(p).upto);
      length += in_these;
      if (first + 64 >= p.B) break;
    }
    before = length - in_these;
    // (the grid is a multiple of eight)
    const int die = blockIdx.x & 7, nth = blockIdx.x >> 3, of_die = gridDim.x >> 3;
    if (by_pieces()) {
      const int share = (length + 7) >> 3;
      at = die * share + nth;
      stop = min((die + 1) * share, length);
      step = of_die;
    } else {
      const int wgs = (int)gridDim.x, nth_window = die * of_die + nth;
      window = __builtin_amdgcn_readfirstlane((length + wgs - 1) / wgs);
      const int64_t begin = (int64_t)nth_window * window;
      at = (int)(begin < length ? begin : length);
      stop = (int)(begin + window < length ? begin + window : length);
      step = 0;
    }
  }
  // the next piece of this workgroup, if there is one
  __device__ __forceinline__ bool next(const CutArgs& p, Piece& r) {
    while (at < stop) {
      if (at < before || at >= before + in_these) {   // of other 64 sequences
        before = in_these = 0;
        first = -64;
        do {
          before += in_these;
          first += 64;
          seq = seq_at(p, first + lane);
          in_these = last_lane(count(p).upto);
        } while (at >= before + in_these);
      }
      const Counts c = count(p);
      const int i = __builtin_ctzll(__ballot(at < before + c.upto));   // the sequence that the place lies in
      r.b = first + i;
      r.len = __builtin_amdgcn_readlane(c.s.len, i);
      r.n = __builtin_amdgcn_readlane(c.s.n, i);
      const int unit = __builtin_amdgcn_readlane(c.unit, i), head = __builtin_amdgcn_readlane(c.head, i);
      const int nb = __builtin_amdgcn_readlane(c.s.nb, i), live = __builtin_amdgcn_readlane(c.s.live, i);
      const int rel = at - before - __builtin_amdgcn_readlane(c.upto - c.own, i);
      r.dead = rel >= p.Hkv * head;
      r.count = 1;
      r.begin = r.end = r.index = r.half = 0;
      int taken = step;
      if (__builtin_expect(r.dead, 0)) {
        const int others = p.groups - live, x = rel - p.Hkv * head, u = x / dead_length(p), off = x - u * dead_length(p);
        r.g = u / others;
        r.y = live + u - r.g * others;
        if (!by_pieces()) {
          taken = dead_length(p) - off;
          r.dead = off == 0;   // (the window that has its first place writes it)
        }
      } else if (p.uncut) {
        r.g = live == 1 ? rel : rel / live;
        r.y = rel - r.g * live;
        r.half = SLABS && r.y == live - 1 ? __builtin_amdgcn_readlane(c.s.half, i) : 0;
        r.end = nb;
      } else {
        r.g = rel / head;
        const int in_head = rel - r.g * head;
        r.y = min(in_head / unit, live - 1);
        const int off = in_head - r.y * unit;
        r.half = SLABS && r.y == live - 1 ? __builtin_amdgcn_readlane(c.s.half, i) : 0;
        const int blocks = (nb + r.half) >> r.half;
        if (by_pieces()) {
          // equal pieces, the first ones a block longer
          const int cuts = r.y == live - 1 ? head - (live - 1) * unit : unit, each = nb / cuts, more = nb - each * cuts;
          r.count = cuts;
          r.index = at;
          r.begin = off * each + min(off, more);
          r.end = r.begin + each + (off < more ? 1 : 0);
        } else {
          // a window has at most one cut piece that starts its unit and one that does not
          const int cost = p.piece_cost, block0 = at - off + cost, from = block0 / window, own = (stop - 1) / window;
          taken = min(cost + blocks - off, stop - at);
          r.begin = max(off - cost, 0) << r.half;
          r.end = min((off + taken - cost) << r.half, nb);
          r.count = (block0 + blocks - 1) / window - from + 1;
          r.index = 2 * own + (r.begin == 0 ? 1 : 0);
        }
      }
      // (quotients come from the vector unit: what follows is the same in all lanes)
      r.g = __builtin_amdgcn_readfirstlane(r.g);
      r.y = __builtin_amdgcn_readfirstlane(r.y);
      r.begin = __builtin_amdgcn_readfirstlane(r.begin);
      r.end = __builtin_amdgcn_readfirstlane(r.end);
      r.count = __builtin_amdgcn_readfirstlane(r.count);
      r.index = __builtin_amdgcn_readfirstlane(r.index);
      r.half = __builtin_amdgcn_readfirstlane(r.half);
      at += __builtin_amdgcn_readfirstlane(taken);
      if (r.dead || r.begin < r.end) return true;
    }
    return false;
  }
};

// ----------------------------------------------------------------------------------------- shared steps
// (Form: what a wavefront's lanes hold and its products, paged_forms.h)

// Hides what a row does not see; visible(t): the 32 keys that this lane's row of tile t does.
template <class Form, typename VisibleFn>
__device__ __forceinline__ void hide(float (&s)[Form::RT][Form::NX], VisibleFn&& visible, float c, int lane) {
  const float hidden = c < 0.f ? INFINITY : -INFINITY;   // (times c: below every score)
#pragma unroll
  for (int t = 0; t < Form::RT; ++t) {
    const unsigned vis = visible(t) >> here(Form::first_key(lane));
#pragma unroll
    for (int j = 0; j < Form::NX; ++j) s[t][j] = ((vis >> Form::key_of(j)) & 1u) ? s[t][j] : hidden;
  }
}

// Exponents of the weights under the shifts in use, and the largest of this lane's.
template <class Form>
__device__ __forceinline__ float exponents(const typename Form::State& st, const float (&s)[Form::RT][Form::NX], float (&x)[Form::RT][Form::NX], float c) {
  float most = -INFINITY;
#pragma unroll
  for (int t = 0; t < Form::RT; ++t) {
    const float m = st.m[t];
#pragma unroll
    for (int j = 0; j < Form::NX; ++j) {
      x[t][j] = fmaf(s[t][j], c, -m);
      most = fmaxf(most, x[t][j]);
    }
  }
  return most;
}

// The same where keys are hidden.
template <class Form, typename VisibleFn>
__device__ __forceinline__ float exponents(const typename Form::State& st, const float (&s)[Form::RT][Form::NX], float (&x)[Form::RT][Form::NX], float c,
                                           VisibleFn&& visible, int lane) {
  float most = -INFINITY;
#pragma unroll
  for (int t = 0; t < Form::RT; ++t) {
    const unsigned vis = visible(t) >> here(Form::first_key(lane));
#pragma unroll
    for (int j = 0; j < Form::NX; ++j) {
      x[t][j] = ((vis >> Form::key_of(j)) & 1u) ? fmaf(s[t][j], c, -st.m[t]) : -INFINITY;
      most = fmaxf(most, x[t][j]);
    }
  }
  return most;
}

// Where a score is too far above its row's shift, rare: the rows' shifts move to their running maxima. The scores are formed again for it
// (score(s)): kept until here they would take sixteen registers more than the exponents made of them.
template <class Form, typename ScoreFn>
__device__ __forceinline__ void settle(typename Form::State& st, float (&x)[Form::RT][Form::NX], float most, float c, ScoreFn&& score) {
  if (__builtin_expect(!__any(most > kLazyLog2), 1)) return;
  float s[Form::RT][Form::NX];
  score(s);
#pragma unroll
  for (int t = 0; t < Form::RT; ++t) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < Form::NX; ++j) top = fmaxf(top, s[t][j] * c);
    const float moved = fmaxf(st.m[t], Form::row_max(top));
    Form::rescale(st, t, __builtin_amdgcn_exp2f(st.m[t] - moved));
    st.m[t] = moved;
#pragma unroll
    for (int j = 0; j < Form::NX; ++j) x[t][j] = fmaf(s[t][j], c, -moved);
  }
}

// Weights are rounded to bf16, which is what the matrix cores take; their sum is that of the rounded ones.
template <class Form>
__device__ __forceinline__ void weigh(const float (&x)[Form::RT][Form::NX], u32x4 (&w)[Form::RT][Form::NX / 8]) {
#pragma unroll
  for (int t = 0; t < Form::RT; ++t)
#pragma unroll
    for (int j = 0; j < Form::NX; j += 2) {
      const bf16x2 two = {(__bf16)__builtin_amdgcn_exp2f(x[t][j]), (__bf16)__builtin_amdgcn_exp2f(x[t][j + 1])};
      w[t][j >> 3][(j & 7) >> 1] = __builtin_bit_cast(unsigned, two);
    }
}

// ---------------------------------------------------------------------------------------------- kernel

// A partial slot: sums in the order in which lanes hold them, [row tile][quad][lane] quads of channels (a store instruction writes a
// kilobyte in a row), behind them the rows' shifts and sums.
template <class Form>
__device__ __forceinline__ int64_t slot_floats(int rows) { return (int64_t)rows * (Form::HEAD_DIM + 2); }
template <class Form>
__device__ __forceinline__ int quad_at(int tile, int quad, int lane) { return ((tile * Form::QUADS + quad) * 64 + lane) * 4; }

__device__ __forceinline__ void put_quad(void* out, bool bf16, int64_t at, f32x4 val) {
  if (bf16) {
    bf16x4 pk;
#pragma unroll
    for (int j = 0; j < 4; ++j) pk[j] = (__bf16)val[j];
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(out) + at) = pk;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = val;
  }
}

// Where 64 blocks lie, one a lane: the bases of codes and scales, or of the two pages (in which a half block is all of its page).
template <bool WIDE>
struct Places {
  uint64_t base[2];
  unsigned vis;

  __device__ __forceinline__ unsigned vis_at(int i) const { return __builtin_amdgcn_readlane(vis, i); }
  __device__ __forceinline__ BlockPlace<WIDE> at(int i) const {
    GlobalBytes b[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      b[k] = (GlobalBytes)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(base[k] >> 32), i) << 32 | (unsigned)__builtin_amdgcn_readlane((int)base[k], i));
    if constexpr (WIDE) return {{b[0]}, {b[1]}};
    else return {{b[0], b[1]}, {b[0], b[1]}};
  }
};

// WIDE: a page holds a block's 32 keys (pages of 16 keys: a block's halves lie on two).
template <class Form, int WAVES, bool WIDE>
__global__ __launch_bounds__(64 * WAVES, WAVES * paged_resident(WAVES, Form::HEAD_DIM, Form::ROWS == 16) / 4)
void tree_attn_paged_kernel(const PagedParams) {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int D = Form::HEAD_DIM, RT = Form::RT, QUADS = Form::QUADS;
  __shared__ f32x4 merge_o[WAVES][RT * QUADS][64];
  __shared__ float2 merge_ml[WAVES][RT][64];
  {   // (a word of each 64 bytes of the arguments: they come from afar, here all at once instead of line by line where they are used. 0.3 us)
    typedef const __attribute__((address_space(4))) unsigned* Words;
    const unsigned line1 = ((Words)p)[16], line2 = ((Words)p)[32], line3 = ((Words)p)[48];
    static_assert(sizeof(PagedParams) > 192 && sizeof(PagedParams) <= 256, "four lines");
    asm volatile("" :: "s"(line1), "s"(line2), "s"(line3));
  }
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  using Cuts = Cutter<(Form::ROWS > 16), (D == 128 && Form::ROWS == 32)>;
  Cuts cutter(cut_args(p), threadIdx.x & 63);
  Piece piece;
  for (bool again = false; cutter.next(cut_args(p), piece); again = true) {
  if (again) __syncthreads();   // the merge buffers are used again
  const int lane = (int)here(threadIdx.x & 63);   // (what is made of it is made for every piece)
  const int b = piece.b, g = piece.g, y = piece.y, L = piece.len, n = piece.n;
  const int ws_shift = piece.half ? 0 : p->ws_shift;
  const int WS = 1 << ws_shift, KW = WAVES >> ws_shift;   // row slabs, wavefronts that split a slab's keys
  const int slab = wave & (WS - 1), kp = wave >> ws_shift;
  const int row0 = y * p->rows_per_group + slab * Form::ROWS;
  if (piece.begin == 0 && threadIdx.x == 0) p->cuts[(b * p->groups + y) * p->Hkv + g] = make_int2(piece.index, piece.count == 1 ? 0 : cutter.by_pieces() ? piece.count : -piece.count);

  // rows that belong to no node; of a unit that was cut the others write them that join its pieces
  if (piece.count == 1 && (piece.dead || piece.half)) {
    const int from = piece.dead ? 0 : Form::ROWS, pieces = D / (p->out_bf16 ? 8 : 4);
    for (int i = threadIdx.x; i < (p->rows_per_group - from) * pieces; i += 64 * WAVES) {
      const int r = i / pieces, rr = y * p->rows_per_group + from + r;
      if (rr >= p->N * p->G) break;
      const int node = (int)div_rcp((unsigned)rr, (unsigned)p->G, p->g_rcp);
      const int64_t row = ((int64_t)b * p->N + node) * p->Hq + g * p->G + (rr - node * p->G);
      *reinterpret_cast<u32x4*>(static_cast<char*>(p->out) + (row * pieces + (i - r * pieces)) * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    if (piece.dead) continue;
  }

  struct RowInfo { bool exists, valid; int node; int64_t out; };
  auto row_info = [&](int t) {
    RowInfo ri;
    const int rr = row0 + Form::TILE * t + Form::row(lane);
    ri.node = (int)div_rcp((unsigned)rr, (unsigned)p->G, p->g_rcp);
    ri.exists = rr < p->N * p->G;
    ri.valid = ri.exists && ri.node < n;
    ri.out = ((int64_t)b * p->N + ri.node) * p->Hq + g * p->G + (rr - ri.node * p->G);
    return ri;
  };

  typename Form::State st;
  Form::clear(st, kNoShift);

  const int tree_blocks = (n + kBlockKeys - 1) / kBlockKeys;   // the first blocks of a unit
  int blk = piece.begin + kp;                                  // neighbouring wavefronts take neighbouring blocks
  if (row0 < n * p->G && blk < piece.end) {
    // the wavefront's places of the prefix: at, at + KW, .. (place i: keys 32 i ..)
    const int P = 1 << p->page_shift;
    const typename Form::Offsets offsets = Form::template offsets<WIDE>(lane, P);
    int at = blk;
    while (at < tree_blocks) at += KW;
    at -= tree_blocks;
    const int end = piece.end - tree_blocks;
    const bool any_prefix = at < end;
    const int turns = any_prefix ? (end - 1 - at) / KW : 0;   // blocks, less one
    // Where blocks lie is found for 64 of them at a time, one a lane, and read from there block by block: scalar bases, to which a
    // lane adds its own places. (Scalar code for one block each turn took about thirty instructions of it, in their order before the others'.)
    using Block = BlockPlace<WIDE>;
    Places<WIDE> places{};
    uint64_t whole = 0;   // of which all 32 keys are there
    auto find = [&](int first) {
      const unsigned t0 = (unsigned)(at + min(first + lane, turns) * KW) * kBlockKeys;
      const int32_t* table = p->table + b * p->table_stride;
      const char* pool = p->pages + (int64_t)g * page_head_bytes(D, P);
      places.vis = ~0u >> (32 - min(L - (int)t0, 32));   // bit t: key t is there
#pragma unroll
      for (int half = 0; half < Block::HALVES; ++half) {
        const unsigned id = (unsigned)table[min(t0 + 16 * half, (unsigned)L - 1) >> p->page_shift], good = id < (unsigned)p->n_pages;
        if (!good) places.vis &= WIDE ? 0u : half == 0 ? 0xffff0000u : 0x0000ffffu;
        const unsigned in_page = (t0 + 16 * half) & (unsigned)(P - 1);
        const uint64_t page = (uint64_t)(uintptr_t)pool + (good ? (uint64_t)id * p->page_stride : 0u);
        places.base[WIDE ? 0 : half] = page + in_page * (WIDE ? D / 2 : 0);
        if (WIDE) places.base[1] = page + in_page;
      }
      whole = __ballot(places.vis == ~0u);
    };
    int nth = 2;   // the place that is read next

    typename Form::Keys keys{}, k_other;
    typename Form::Values v_this{}, v_other;
    Block block{}, block_next{};
    unsigned vis_here = 0, vis_next = 0;
    if (any_prefix) {
      find(0);
      block = places.at(0);
      vis_here = places.vis_at(0);
      block_next = places.at(1);
      vis_next = places.vis_at(1);
      Form::load_keys(keys, block, offsets, lane, P);
    }
    u32x4 q_row[RT][Form::PIECES];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const RowInfo ri = row_info(t);
#pragma unroll
      for (int i = 0; i < Form::PIECES; ++i)
        q_row[t][i] = ri.valid ? *reinterpret_cast<const u32x4*>(p->q + (ri.out * D + Form::piece_channel(i, lane)) * 2) : u32x4{0u, 0u, 0u, 0u};
    }

    u32x4 w[RT][Form::NX / 8];
    // ---- blocks of the tree
    for (; blk < min(tree_blocks, piece.end); blk += KW) {
      const int t0 = blk * kBlockKeys;
      const int64_t row = (int64_t)p->Hkv * D * 2;
      const char* kr = p->k_tree + ((int64_t)b * p->N * p->Hkv + g) * (D * 2);
      const char* vr = p->v_tree + ((int64_t)b * p->N * p->Hkv + g) * (D * 2);
      typename Form::TreeKeys tree_keys;
      typename Form::TreeValues values;
      uint64_t tree_mask[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const RowInfo ri = row_info(t);
        tree_mask[t] = ri.valid ? p->mask[b * p->N + ri.node] : 0ull;
      }
      Form::load_tree(tree_keys, values, kr, vr, row, t0, n - 1, lane);
      constexpr int VALUE_WORDS = sizeof(values.v[0]) / 4;
      unsigned wild = 0;
#pragma unroll
      for (int j = 0; j < Form::NX; ++j)
#pragma unroll
        for (int i = 0; i < VALUE_WORDS; ++i) wild |= has_wild(values.v[j][i]);
      // A weight of zero does not keep NaN and infinity out of a product. Where the tree's values hold any, they are taken out
      // here and added below to the rows that see them.
      const bool any_wild = __any(wild != 0);
      if (__builtin_expect(any_wild, 0)) {
#pragma unroll
        for (int j = 0; j < Form::NX; ++j)
#pragma unroll
          for (int i = 0; i < VALUE_WORDS; ++i) values.v[j][i] &= ~wild_halves(values.v[j][i]);
      }
      const unsigned there = n - t0 >= kBlockKeys ? ~0u : (1u << (n - t0)) - 1u;
      auto visible = [&](int t) { return (unsigned)(tree_mask[t] >> t0) & there; };
      float s[RT][Form::NX], x[RT][Form::NX];
      auto score = [&](float (&s)[RT][Form::NX]) {
        Form::score_tree(s, tree_keys, q_row);
        hide<Form>(s, visible, p->c, lane);
      };
      Form::score_tree(s, tree_keys, q_row);
      settle<Form>(st, x, exponents<Form>(st, s, x, p->c, visible, lane), p->c, score);
      weigh<Form>(x, w);
      Form::accumulate_tree(st, w, values);
      if (__builtin_expect(any_wild, 0)) {
#pragma unroll 1
        for (int key = 0; key < kBlockKeys; ++key) {
          if (!((there >> key) & 1u)) break;
          const char* src = vr + (t0 + key) * row;
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const float weight = Form::weight_of(w[t], key, lane);
            if (!((visible(t) >> key) & 1u)) continue;
#pragma unroll
            for (int q = 0; q < QUADS; ++q)
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                const unsigned w2 = *reinterpret_cast<const unsigned*>(src + 2 * (Form::channel(q, lane) + k));
                const unsigned odd = wild_halves(w2);
                if (odd & 0xffffu) Form::add_to(st, t, q, k, weight * __builtin_bit_cast(float, w2 << 16));
                if (odd >> 16) Form::add_to(st, t, q, k + 1, weight * __builtin_bit_cast(float, w2 & 0xffff0000u));
              }
          }
        }
      }
    }

    // ---- blocks of the prefix. A turn forms the weights and sums of one block and the scores of the next: its products do not wait
    // for the exponentials, nor these for them. Its values and the keys of the block after it were asked for a turn ahead. The first turn
    // has no block yet (weights of zero: the scores' code stands once), the last one forms its own scores again, for nobody.
    if (any_prefix) {
      typename Form::Query q;
      float x[RT][Form::NX];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        Form::split(q, t, q_row[t], lane);
#pragma unroll
        for (int j = 0; j < Form::NX; ++j) x[t][j] = -INFINITY;
      }
      const float c = p->c;
      unsigned vis_this = ~0u;   // (values of zero, scales of 2^-127)
      // (two turns stand in each loop, each with registers of its own for what it asks for: copied from one set to another, loads would
      // be waited for in the turn that asks for them)
      auto turn = [&](auto some_hidden, typename Form::Keys& k_this, typename Form::Keys& k_third, typename Form::Values& v_this, typename Form::Values& v_next) {
        constexpr bool SOME_HIDDEN = decltype(some_hidden)::value;
        Form::load_values(v_next, block, offsets, lane);
        const unsigned vis = vis_here;
        block = block_next;
        Form::load_keys(k_third, block, offsets, lane, P);
        block_next = places.at(nth & 63);
        ++nth;
        if constexpr (SOME_HIDDEN) {
          vis_here = vis_next;
          vis_next = places.vis_at((nth - 1) & 63);
          if ((nth & 63) == 0) find(nth);
        }
        weigh<Form>(x, w);
        __builtin_amdgcn_sched_barrier(0);
        float s[RT][Form::NX];
        Form::score(s, k_this, q);
        __builtin_amdgcn_sched_barrier(0);
        if (SOME_HIDDEN && vis_this != ~0u) Form::mask_values(v_this, vis_this, lane);
        float most;
        Form::accumulate(st, w, v_this, [&] {   // (the exponents between its products: whether they are too large is known when they end)
          most = SOME_HIDDEN ? exponents<Form>(st, s, x, c, [&](int) { return vis; }, lane) : exponents<Form>(st, s, x, c);
        });
        settle<Form>(st, x, most, c, [&](float (&again)[RT][Form::NX]) {
          Form::score(again, k_this, q);
          if (SOME_HIDDEN) hide<Form>(again, [&](int) { return vis; }, c, lane);
        });
        if (SOME_HIDDEN) vis_this = vis;
      };
      for (int left = turns + 2;;) {
        // turns that need not look whether all keys are there: as many as places with all of theirs follow the whole ones in work
        if ((vis_this & vis_here & vis_next) == ~0u) {
          const uint64_t others = ~(whole >> (nth & 63));   // (63 at most: the place behind the 64th is not in `whole`)
          const int run = min(min(others ? (int)__builtin_ctzll(others) : 64, 63 - (nth & 63)), left) >> 1;
          left -= 2 * run;
          for (int i = 0; i < run; ++i) {
            turn(std::false_type{}, keys, k_other, v_this, v_other);
            turn(std::false_type{}, k_other, keys, v_other, v_this);
          }
          if (left == 0) break;
        }
        turn(std::true_type{}, keys, k_other, v_this, v_other);
        if (--left == 0) break;
        turn(std::true_type{}, k_other, keys, v_other, v_this);
        if (--left == 0) break;
      }
    }
  }
  p = fresh(p);

  // ---- the key-splitting wavefronts of a slab meet in LDS; each writes its share of the quads
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    merge_ml[wave][t][lane] = make_float2(st.m[t], Form::row_sum(st, t));
#pragma unroll
    for (int q = 0; q < QUADS; ++q) merge_o[wave][t * QUADS + q][lane] = Form::quad(st, t, q);
  }
  __syncthreads();
  constexpr int SHARE = RT * QUADS >= WAVES ? RT * QUADS / WAVES : 1;   // quads at a time
  for (int at = kp * SHARE; at < RT * QUADS; at += KW * SHARE) {
    const int t = at / QUADS, q0 = at - t * QUADS;
    float mm = kNoShift;
#pragma unroll 4
    for (int k = 0; k < KW; ++k) mm = fmaxf(mm, merge_ml[slab + k * WS][t][lane].x);   // (four or eight)
    float l_row = 0.f;
    f32x4 o[SHARE];
#pragma unroll
    for (int j = 0; j < SHARE; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < KW; ++k) {   // in wavefront order: the same bits every time
      const float2 ml = merge_ml[slab + k * WS][t][lane];
      const float a = __builtin_amdgcn_exp2f(ml.x - mm);
      l_row += ml.y * a;
#pragma unroll
      for (int j = 0; j < SHARE; ++j) o[j] += merge_o[slab + k * WS][at + j][lane] * a;
    }
    const RowInfo ri = row_info(t);
    if (!ri.exists) continue;
    if (piece.count == 1) {
      const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;
#pragma unroll
      for (int j = 0; j < SHARE; ++j)
        put_quad(p->out, p->out_bf16, ri.out * D + Form::channel(q0 + j, lane), ri.valid ? o[j] * inv : f32x4{0.f, 0.f, 0.f, 0.f});
    } else if (ri.valid) {   // (the join reads no others)
      float* part = p->part + piece.index * slot_floats<Form>(p->rows_per_group);
      const int tile = slab * RT + t;
      if (Form::first_key(lane) == 0 && q0 == 0)
        *reinterpret_cast<float2*>(part + (int64_t)p->rows_per_group * D + 2 * (Form::TILE * tile + Form::row(lane))) = make_float2(mm, l_row);
#pragma unroll
      for (int j = 0; j < SHARE; ++j) *reinterpret_cast<f32x4*>(part + quad_at<Form>(tile, q0 + j, lane)) = o[j];
    }
  }
  }
}

// Joins the pieces of the units that were cut: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s. A wavefront has a quad as the pieces'
// wavefronts left it: four channels of a row a lane.
template <class Form>
__global__ __launch_bounds__(256) void tree_attn_paged_join_kernel(const PagedParams p) {
  constexpr int D = Form::HEAD_DIM;
  const int g = blockIdx.y, y = blockIdx.z % p.groups, b = blockIdx.z / p.groups;
  const int2 cut = p.cuts[(b * p.groups + y) * p.Hkv + g];
  int nodes = p.cut.n_nodes[b];
  asm volatile("" : "+s"(nodes));   // (asked for together with the other)
  if (cut.y == 0) return;
  const int lane = threadIdx.x & 63, item = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int quad = item % Form::QUADS, tile = item / Form::QUADS;
  const int lr = Form::TILE * tile + Form::row(lane), rr = y * p.rows_per_group + lr;
  if (lr >= p.rows_per_group || rr >= p.N * p.G) return;
  const int node = (int)div_rcp((unsigned)rr, (unsigned)p.G, p.g_rcp);
  const int n = min(max(nodes, 0), p.N);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (node < n) {
    const int64_t slot = slot_floats<Form>(p.rows_per_group);
    const float* o_at = p.part + quad_at<Form>(tile, quad, lane);
    const float* ml_at = p.part + (int64_t)p.rows_per_group * D + 2 * lr;
    const int pieces = abs(cut.y);
    float M = kNoShift, sum = 0.f;
    for (int s0 = 0; s0 < pieces; s0 += 8) {   // in order: the same bits every time
      float2 ml[8];
      f32x4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // (windows have two slots each: a unit's first piece is in the second one of its window, the others in the first ones of theirs)
        const int s = min(s0 + k, pieces - 1);
        const int64_t at = (int64_t)(cut.x + s + (cut.y < 0 && s > 0 ? s - 1 : 0)) * slot;
        ml[k] = *reinterpret_cast<const float2*>(ml_at + at);
        o[k] = *reinterpret_cast<const f32x4*>(o_at + at);
      }
      float mx = M;
#pragma unroll
      for (int k = 0; k < 8; ++k) mx = fmaxf(mx, ml[k].x);
      const float a = __builtin_amdgcn_exp2f(M - mx);
      acc *= a;
      sum *= a;
      M = mx;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (s0 + k >= pieces) break;
        const float wgt = __builtin_amdgcn_exp2f(ml[k].x - M);
        sum += wgt * ml[k].y;
        acc += wgt * o[k];
      }
    }
    acc *= sum == 0.f ? 0.f : 1.0f / sum;
  }
  put_quad(p.out, p.out_bf16, (((int64_t)b * p.N + node) * p.Hq + g * p.G + (rr - node * p.G)) * D + Form::channel(quad, lane), acc);
}

template <class Form, int WAVES, bool WIDE>
void launch(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  // a multiple of eight: workgroup w takes places w / 8, one grid's eighth further, .. of die w % 8's share
  const int wgs = pl.max_pieces < pl.resident ? pl.max_pieces : pl.resident;
  hipLaunchKernelGGL((tree_attn_paged_kernel<Form, WAVES, WIDE>), dim3((unsigned)((wgs + 7) / 8 * 8)), dim3(64 * WAVES), 0, stream, p);
  if (!pl.may_cut) return;
  const int rows = pl.rows_per_group < p.N * p.G ? pl.rows_per_group : p.N * p.G;
  hipLaunchKernelGGL((tree_attn_paged_join_kernel<Form>), dim3((unsigned)((rows + Form::TILE - 1) / Form::TILE * (Form::QUADS / 4)), (unsigned)p.Hkv,
                                                               (unsigned)(p.B * pl.groups)), dim3(256), 0, stream, p);
}

template <int D, bool WIDE>
void launch_rows(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  if (pl.rows_per_wave == 16) pl.waves == 4 ? launch<Form16<D>, 4, WIDE>(pl, p, stream) : launch<Form16<D>, 8, WIDE>(pl, p, stream);
  else if (pl.rows_per_wave == 32) pl.waves == 4 ? launch<Form32<D, 1>, 4, WIDE>(pl, p, stream) : launch<Form32<D, 1>, 8, WIDE>(pl, p, stream);
  else if constexpr (D == 64) pl.waves == 4 ? launch<Form32<64, 2>, 4, WIDE>(pl, p, stream) : launch<Form32<64, 2>, 8, WIDE>(pl, p, stream);
}

}  // namespace

extern "C" size_t fspad_tree_attn_paged_workspace_bytes(const fspad_paged_desc* desc) {
  if (!desc || check_paged_attn(*desc) != FSPAD_OK) return 0;
  return plan_paged(*desc).workspace_bytes;
}

extern "C" fspad_status fspad_tree_attn_paged(const fspad_paged_desc* desc, const void* q, const void* k_tree, const void* v_tree,
                                              const void* pages, const int32_t* block_table, const int32_t* kv_len,
                                              const int32_t* n_nodes, const uint64_t* anc_mask, void* out, void* workspace,
                                              size_t workspace_bytes, void* hip_stream) {
  if (!desc) return FSPAD_ERR_NULL;
  const fspad_paged_desc& d = *desc;
  if (const fspad_status st = check_paged_attn(d)) return st;
  if (!q || !k_tree || !v_tree || !pages || !block_table || !kv_len || !n_nodes || !anc_mask || !out) return FSPAD_ERR_NULL;
  if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)pages | (uintptr_t)out) & 15) return FSPAD_ERR_SHAPE;
  const float c = (d.softmax_scale == 0.f ? 1.0f / sqrtf((float)d.head_dim) : d.softmax_scale) * 1.44269504088896340736f;
  if (!(fabsf(c) >= FLT_MIN && fabsf(c) <= FLT_MAX)) return FSPAD_ERR_SHAPE;
  const PagedPlan pl = plan_paged(d);
  if (!workspace || workspace_bytes < pl.workspace_bytes || ((uintptr_t)workspace & 15)) return FSPAD_ERR_WORKSPACE;
  PagedParams p{};
  p.q = static_cast<const char*>(q); p.k_tree = static_cast<const char*>(k_tree); p.v_tree = static_cast<const char*>(v_tree);
  p.pages = static_cast<const char*>(pages); p.table = block_table; p.mask = anc_mask;
  p.out = out; p.cuts = static_cast<int2*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.cuts_bytes);
  p.page_stride = (uint32_t)d.page_stride; p.table_stride = d.table_stride;
  p.B = d.batch; p.N = d.n_nodes_max; p.Hq = d.n_q_heads; p.Hkv = d.n_kv_heads; p.G = d.n_q_heads / d.n_kv_heads;
  p.page_shift = log2_of(d.page_tokens); p.n_pages = d.n_pages;
  p.g_rcp = reciprocal(p.G);
  p.ws_shift = log2_of(pl.WS); p.rows_per_group = pl.rows_per_group; p.groups = pl.groups;
  p.out_bf16 = d.out_dtype == FSPAD_BF16;
  p.cut = {kv_len, n_nodes, p.B, p.N, p.G, p.Hkv, log2_of(pl.rows_per_group), p.ws_shift, p.groups, d.max_kv_len, pl.resident, pl.max_pieces,
           pl.least_blocks, pl.whole_blocks, pl.piece_cost, pl.join_cost, pl.dead_cost, pl.lines, !pl.may_cut, d.workgroups};
  p.c = c;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const bool wide = d.page_tokens >= kBlockKeys;
  if (d.head_dim == 128) wide ? launch_rows<128, true>(pl, p, stream) : launch_rows<128, false>(pl, p, stream);
  else wide ? launch_rows<64, true>(pl, p, stream) : launch_rows<64, false>(pl, p, stream);
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}
