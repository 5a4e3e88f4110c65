// Tree-masked attention over a paged 4-bit cache (arXiv 2408.15562, Preliminaries, validation phase, as fspad_attn.hip; the
// cache format is in include/fspad.h). gfx950 (CDNA4) only.
//
// One pass over the keys with a running shift and sum per query row. A wavefront owns up to 64 query rows (16-row tiles) of one
// kv head and takes 32-key blocks of K and V from the pages straight into registers, 4 bits an entry. The layout of the pages is that
// of the operands (lane (col, g4): col = lane % 16, g4 = lane / 16):
//   S^T = K Q^T    on the block-scaled products (v_mfma_scale_f32_16x16x128_f8f6f4), which take K's codes and scales as they are: a
//                  lane holds one block of 32 channels of key col, 16 bytes and a scale byte. They have no bf16 operand; a query row
//                  is two fp8 ones instead (split_q), whose sum it is: D = 128 in two products, D = 64 in one, K's 64 channels twice
//                  in its 128. As many clocks as bf16 products take, a quarter to half of the instructions, and nothing to convert:
//   O^T += V^T P^T V's scales run along the channels, not along the keys that are summed over, so V becomes bf16
//                  (v_cvt_scalef32_pk_bf16_fp4: two entries and their block's scale in one instruction, exact). A lane holds
//                  D/16 channels of the keys 4 g4 .. 4 g4 + 3 and 16 more, those whose scores S^T leaves in it: the weights
//                  never leave the lane they arise in, and a page of 16 keys is half a block for all lanes alike. The 8 x D/16 entries
//                  turn from key order to channel order two bytes at a time (v_perm_b32).
//
// How a call is cut is decided on the device, from lengths it alone knows (piece_plan): a unit, 64 query rows or less of one kv head of one
// sequence, is one workgroup's or is cut along its keys into equal pieces, a workgroup each. A whole unit goes straight to `out`; of
// the others every piece leaves its un-normalised sums in the workspace and a second kernel joins them.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"
#include "paged_plan.h"
#include "stream_gemm.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef const __attribute__((address_space(4))) int32_t* ScalarI32;
typedef const __attribute__((address_space(1))) char* GlobalBytes;

struct PagedParams {
  const char* q;
  const char* k_tree;
  const char* v_tree;
  const char* pages;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* n_nodes;
  const uint64_t* mask;
  void* out;
  int2* cuts;       // per unit: first partial slot and number of pieces (0: the unit is complete in `out`)
  float* part;      // partial slots, one for every piece
  int64_t table_stride;
  uint32_t page_stride;
  int32_t B, N, Hq, Hkv, G, page_shift, n_pages, max_kv_len;
  uint32_t g_rcp;   // reciprocal(G)
  int32_t ws_shift, rows_shift, rows_per_group, groups, max_pieces, resident, least_blocks, whole_blocks, piece_cost, forced, out_bf16;
  float c;          // softmax scale * log2(e)
};

// The arguments where the launch left them. What only a segment's start or end needs is fetched there, through a pointer that the
// compiler takes for another one each time: kept in scalar registers for the length of a stream, arguments displaced what the stream needs.
typedef const __attribute__((address_space(4))) PagedParams* Args;
__device__ __forceinline__ Args fresh(Args p) {
  asm volatile("" : "+s"(p));
  return p;
}

// A lane's number, as it stands here: what is made of it is not made ahead of a loop and kept. (An offset that was widened to 64 bits there
// would be added to every address by instructions of its own, instead of by the load.)
__device__ __forceinline__ unsigned here(unsigned offset) {
  asm volatile("" : "+v"(offset));
  return offset;
}

// The shift of a row moves only when a score exceeds it by more than this (log2 units): weights stay below 2^8, which fp32 sums
// and bf16 weights hold without loss, and accumulators are rescaled almost never after the first blocks.
constexpr float kLazyLog2 = 8.0f;
constexpr float kNoShift = -FLT_MAX;   // below every score: the first visible one moves it

// ------------------------------------------------------------------------------------------------ plan

// What a sequence is made of: `live` row groups of nb blocks each per kv head, the others without nodes (they write zeros).
struct SeqShape {
  int len, n, live, nb;
};
__device__ __forceinline__ int2 seq_at(Args p, int b) { return b < p->B ? make_int2(p->kv_len[b], p->n_nodes[b]) : make_int2(0, 0); }
__device__ __forceinline__ SeqShape shape_of(Args p, int2 seq) {
  SeqShape s;
  s.len = min(max(seq.x, 0), p->max_kv_len);
  s.n = min(max(seq.y, 0), p->N);
  s.live = (s.n * p->G + p->rows_per_group - 1) >> p->rows_shift;
  s.nb = s.live > 0 ? (s.len + kBlockKeys - 1) / kBlockKeys + (s.n + kBlockKeys - 1) / kBlockKeys : 0;
  return s;
}

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

// Blocks of a piece, at most, for `blocks` blocks in `units` units of `longest` blocks at most. Pieces of one round (as many as the
// device holds workgroups at once), if the units can be cut into so few, take as long as the longest of them; smaller ones in
// several rounds share the device better and pay for starting and ending more often.
__device__ __forceinline__ int piece_length(Args p, int blocks, int units, int longest) {
  const float slots = (float)(p->max_pieces - p->B * p->Hkv * p->groups);   // the sum of ceil(nb / len) is at most S / len + units
  if (p->forced > 0) return max((int)ceilf((float)blocks / slots) + 1, 1);
  if (longest <= p->whole_blocks) return max(longest, 1);
  const float R = (float)p->resident, S = (float)blocks, U = (float)units, piece_cost = (float)p->piece_cost;
  float len = (float)longest, cost = S / R + fmaxf(U / R, 1.0f) * piece_cost + 0.5f * len;   // whole units
  if (units < p->resident) {
    const float one = fminf(ceilf(S / (R - U)), ceilf(len / floorf(R / U)));   // either way there are at most R pieces
    len = fminf(len, one);
    cost = len + piece_cost;
  }
  const float many = ceilf(__builtin_sqrtf(2.0f * piece_cost * S / R));
  if ((S + (S / many + 0.5f * U) * piece_cost) / R + 0.5f * many < cost) len = fminf(len, many);
  len = fmaxf(len, ceilf(S / slots) + 1.0f);
  return max((int)len, p->least_blocks);
}

// How the call is cut, and the pieces of this workgroup. Pieces are numbered sequence by sequence, head by head, group by group, along the
// keys; workgroups eight apart, which share a die and its L2 cache, take neighbouring ones.
struct Piece {
  int b, g, y, len, n, begin, end, index, count;   // blocks [begin, end) of a unit; index: its slot; count: pieces of the unit
  bool dead;
};
struct Cutter {
  Args p;
  int lane, most, places;   // blocks of a piece, at most; pieces in all
  int2 seq;                 // 64 sequences at a time, one a lane, from `first` on: length and nodes
  int first, before, in_these;   // places before theirs, and theirs

  struct Counts {
    SeqShape s;
    int cuts, own, upto;
  };
  __device__ __forceinline__ Counts count() const {
    Counts c;
    c.s = shape_of(p, seq);
    c.cuts = (c.s.nb + most - 1) / most;
    c.own = first + lane < p->B ? p->Hkv * (c.s.live * c.cuts + p->groups - c.s.live) : 0;
    c.upto = wave_sum_upto(c.own);
    return c;
  }
  __device__ __forceinline__ Cutter(Args args, int lane_) : p(args), lane(lane_) {
    seq = seq_at(p, lane);
    int blocks = 0, units = 0, longest = 0;
    for (first = 0;;) {
      const SeqShape s = shape_of(p, seq);
      const int of = p->Hkv * s.live;
      blocks += last_lane(wave_sum_upto(of * s.nb));
      units += last_lane(wave_sum_upto(of));
      longest = max(longest, last_lane(wave_max_upto(s.nb)));
      first += 64;
      if (first >= p->B) break;
      seq = seq_at(p, first + lane);
    }
    most = __builtin_amdgcn_readfirstlane(piece_length(p, blocks, units, longest));
    places = 0;
    for (first = 0;; first += 64) {
      if (p->B > 64) seq = seq_at(p, first + lane);
      in_these = last_lane(count().upto);
      places += in_these;
      if (first + 64 >= p->B) break;
    }
    before = places - in_these;
  }
  // place `at` < places
  __device__ __forceinline__ Piece piece(int at) {
    if (at < before || at >= before + in_these) {   // of other 64 sequences
      before = in_these = 0;
      first = -64;
      do {
        before += in_these;
        first += 64;
        seq = seq_at(p, first + lane);
        in_these = last_lane(count().upto);
      } while (at >= before + in_these);
    }
    const Counts c = count();
    Piece r{};
    const int i = __builtin_ctzll(__ballot(at < before + c.upto));   // the sequence that the place lies in
    r.b = first + i;
    r.len = __builtin_amdgcn_readlane(c.s.len, i);
    r.n = __builtin_amdgcn_readlane(c.s.n, i);
    r.count = __builtin_amdgcn_readlane(c.cuts, i);
    r.index = at;
    const int nb = __builtin_amdgcn_readlane(c.s.nb, i), live = __builtin_amdgcn_readlane(c.s.live, i);
    const int rel = at - before - __builtin_amdgcn_readlane(c.upto - c.own, i), heads = p->Hkv * live * r.count;
    r.dead = rel >= heads;
    if (__builtin_expect(r.dead, 0)) {
      const int others = p->groups - live, x = rel - heads;
      r.g = x / others;
      r.y = live + x - r.g * others;
      r.count = 1;
    } else {
      const int u = rel / r.count, part = rel - u * r.count;
      r.g = u / live;
      r.y = u - r.g * live;
      // equal pieces, the first ones a block longer
      const int each = nb / r.count, more = nb - each * r.count;
      r.begin = part * each + min(part, more);
      r.end = r.begin + each + (part < more ? 1 : 0);
    }
    // (quotients come from the vector unit: what follows is the same in all lanes)
    r.g = __builtin_amdgcn_readfirstlane(r.g);
    r.y = __builtin_amdgcn_readfirstlane(r.y);
    r.begin = __builtin_amdgcn_readfirstlane(r.begin);
    r.end = __builtin_amdgcn_readfirstlane(r.end);
    return r;
  }
};

// -------------------------------------------------------------------------------------------- operands

template <int QT, int D>
struct RowState {
  static constexpr int DT = D / 16;
  f32x4 o[QT][DT];   // O^T: lane (col, g4), entry i <-> row 16 t + col, channel DT (4 g4 + i) + e
  float m[QT];       // shift in use (log2 units): within kLazyLog2 of the running maximum
  float l[QT];       // sum of the rounded weights
};

// (key 2i, key 2i+1) of one channel from (channel, next channel) of the two keys
__device__ __forceinline__ unsigned pair_low(unsigned first, unsigned second) { return __builtin_amdgcn_perm(second, first, 0x05040100u); }
__device__ __forceinline__ unsigned pair_high(unsigned first, unsigned second) { return __builtin_amdgcn_perm(second, first, 0x07060302u); }

__device__ __forceinline__ void turn(const unsigned (&x)[8], bf16x8& even, bf16x8& odd) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = pair_low(x[2 * i], x[2 * i + 1]);
    b[i] = pair_high(x[2 * i], x[2 * i + 1]);
  }
  even = __builtin_bit_cast(bf16x8, a);
  odd = __builtin_bit_cast(bf16x8, b);
}

template <int BYTE>
__device__ __forceinline__ unsigned two_values(unsigned codes, float scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
__device__ __forceinline__ unsigned two_values(unsigned codes, float scale, int byte) {   // (byte: a constant once unrolled)
  return byte == 0 ? two_values<0>(codes, scale) : byte == 1 ? two_values<1>(codes, scale) : byte == 2 ? two_values<2>(codes, scale)
                                                                                           : two_values<3>(codes, scale);
}

// The lane's j-th key of a block, less 4 g4.
__device__ constexpr int key_of(int j) { return (j & 3) + 16 * (j >> 2); }

// K and V of a 32-key block of the prefix as they lie in the pages. Keys that are not there (past the length, on a bad page) are
// masked by their scores; their values only have to be finite, which codes are under any scale but 255.
struct __attribute__((packed)) Unaligned { unsigned word; };
struct PagedK {
  u32x4 c[2];
  unsigned scale[2];
};

// Query rows as the block-scaled products take them: row = hi + lo, each fp8 (e4m3, 4 significant bits) times a power of two of the
// row. A bf16 value has 8 significant bits: hi takes the upper four, and what is left of them is a multiple of the value's last
// place, eight at most, which lo holds exactly. With the row's largest magnitude at 128 .. 256 in hi's units (and what is left of it
// below 256 in lo's, 32 times finer) this holds down to 2^-14 of the largest; below that a value is off by 2^-22 of the largest at
// most. Rows with NaN or infinity have the scale that is NaN.
template <int D>
struct SplitQ {
  i32x8 v[D / 64];     // D = 128: hi, lo; D = 64: hi in the first half, lo in the second
  int scale;           // D = 128: hi's in the first byte, lo's in the second

  // x: channels 16 g4 .. + 15 of the row, D = 128 also 64 + 16 g4 .. + 15, bf16 pairs
  __device__ __forceinline__ void split(const u32x4 (&x)[D / 32], int g4) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned w = x[i][k];
        top = max(top, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
      }
    top = max(top, (unsigned)__shfl_xor((int)top, 16));
    top = max(top, (unsigned)__shfl_xor((int)top, 32));
    const int e = max((int)(top >> 7), 13) - 7;                    // hi's scale byte; lo's is 5 less
    const bool wild = top >= 0x7f80u;
    const float to_hi = __builtin_bit_cast(float, (254 - e) << 23);   // 2^(127 - e); e <= 248
    i32x8 hi{}, lo{};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned w = x[i][k];
        const float a = wild ? 0.f : __builtin_bit_cast(float, w << 16) * to_hi, b = wild ? 0.f : __builtin_bit_cast(float, w & 0xffff0000u) * to_hi;
        const int h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        const f32x2 back = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
        const int l = __builtin_amdgcn_cvt_pk_fp8_f32((a - back[0]) * 32.f, (b - back[1]) * 32.f, 0, false);
        const int at = 2 * i + (k >> 1), shift = 16 * (k & 1);
        hi[at] |= (h & 0xffff) << shift;
        lo[at] |= (l & 0xffff) << shift;
      }
    const int s_hi = wild ? 255 : e, s_lo = wild ? 255 : e - 5;
    if constexpr (D == 128) {
      v[0] = hi; v[1] = lo;
      scale = s_hi | s_lo << 8;
    } else {
      v[0] = i32x8{hi[0], hi[1], hi[2], hi[3], lo[0], lo[1], lo[2], lo[3]};
      scale = g4 < 2 ? s_hi : s_lo;   // a lane's scale is that of the products' channels 32 g4 .. + 31
    }
  }
};

template <int D>
struct PagedV {
  unsigned c[D / 16];
  unsigned scale[2];
  float f[8];   // scales of the lane's keys

  __device__ __forceinline__ void ready(unsigned vis, int g4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // (the conversion takes the exponent of its scale: what lies around the byte does not matter)
      const unsigned w = scale[j >> 2];
      f[j] = __builtin_bit_cast(float, (j & 3) == 3 ? w >> 1 : w << (23 - 8 * (j & 3)));
    }
    if (__builtin_expect(vis != ~0u, 0)) {
      const unsigned own = vis >> here(4 * g4);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = ((own >> key_of(j)) & 1u) ? f[j] : 1.0f;
    }
  }
  __device__ __forceinline__ void v_pair(int e2, bf16x8& even, bf16x8& odd) const {
    unsigned x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = D == 128 ? two_values(c[j], f[j], e2) : two_values(c[j >> 1], f[j], 2 * (j & 1) + e2);
    turn(x, even, odd);
  }
};

// Values of a block of the tree's own keys, bf16 (rows past the tree's end repeat its last one and are masked).
template <int D>
struct TreeV {
  unsigned v[8][D / 32];

  __device__ __forceinline__ void v_pair(int e2, bf16x8& even, bf16x8& odd) const {
    unsigned x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[j][e2];
    turn(x, even, odd);
  }
};

// (an exponent of all ones carries into the sign's place when one is added to it)
__device__ __forceinline__ unsigned has_wild(unsigned w) {
  return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
__device__ __forceinline__ unsigned wild_halves(unsigned w) {   // all bits of a half that holds NaN or infinity
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

template <int QT>
using Scores = f32x4[QT][2];   // lane (col, g4), [t][kt][i]: key 16 kt + 4 g4 + i against row 16 t + col

template <int QT, int D>
__device__ __forceinline__ void score_block(Scores<QT>& s, const PagedK& keys, const SplitQ<D> (&q)[QT]) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const u32x4 c = keys.c[kt];
    const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < QT; ++t)
      s[t][kt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q[t].v[0], f32x4{0.f, 0.f, 0.f, 0.f}, 4 /* a: fp4 */, 0 /* b: e4m3 */, 0, (int)keys.scale[kt],
                                                                  0, q[t].scale);
    if constexpr (D == 128) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
        s[t][kt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q[t].v[1], s[t][kt], 4, 0, 0, (int)keys.scale[kt], 1 /* the second byte */, q[t].scale);
    }
  }
}

// The tree's own keys and the query rows as they are.
template <int QT, int D>
__device__ __forceinline__ void score_tree(Scores<QT>& s, const bf16x8 (&k)[2][D / 32], const u32x4 (&q)[QT][D / 32]) {
#pragma unroll
  for (int t = 0; t < QT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[kt][ks], __builtin_bit_cast(bf16x8, q[t][ks]), s[t][kt], 0, 0, 0);
}

// Hides what a row does not see; visible(t): the 32 keys that this lane's row of tile t does.
template <int QT, typename VisibleFn>
__device__ __forceinline__ void hide(Scores<QT>& s, VisibleFn&& visible, float c, int g4) {
  const float hidden = c < 0.f ? INFINITY : -INFINITY;   // (times c: below every score)
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const unsigned vis = visible(t) >> here(4 * g4);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[t][j >> 2][j & 3] = ((vis >> key_of(j)) & 1u) ? s[t][j >> 2][j & 3] : hidden;
  }
}

// Exponents of the weights under the shifts in use, and the largest of this lane's.
template <int QT, int D>
__device__ __forceinline__ float exponents(const RowState<QT, D>& st, const Scores<QT>& s, float (&x)[QT][8], float c) {
  float most = -INFINITY;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float m = st.m[t];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[t][j] = fmaf(s[t][j >> 2][j & 3], c, -m);
      most = fmaxf(most, x[t][j]);
    }
  }
  return most;
}

// Where a score is too far above its row's shift, rare: the rows' shifts move to their running maxima. The scores are formed again for it
// (score(s)): kept until here they would take sixteen registers more than the exponents made of them.
template <int QT, int D, typename ScoreFn>
__device__ __forceinline__ void settle(RowState<QT, D>& st, float (&x)[QT][8], float most, float c, ScoreFn&& score) {
  if (__builtin_expect(!__any(most > kLazyLog2), 1)) return;
  Scores<QT> s;
  score(s);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, s[t][j >> 2][j & 3] * c);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float moved = fmaxf(st.m[t], top);
    const float alpha = __builtin_amdgcn_exp2f(st.m[t] - moved);
    st.m[t] = moved;
    st.l[t] *= alpha;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) st.o[t][e] *= alpha;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[t][j] = fmaf(s[t][j >> 2][j & 3], c, -moved);
  }
}

// Weights are rounded to bf16, which is what the matrix cores take; their sum is that of the rounded ones.
template <int QT>
__device__ __forceinline__ void weigh(const float (&x)[QT][8], bf16x8 (&pf)[QT]) {
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) pf[t][j] = (__bf16)__builtin_amdgcn_exp2f(x[t][j]);
}

template <int QT, int D, typename Values>
__device__ __forceinline__ void accumulate(RowState<QT, D>& st, const bf16x8 (&pf)[QT], const Values& values) {
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
#pragma unroll
  for (int t = 0; t < QT; ++t) st.l[t] += __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0)[0];   // (all entries equal)
#pragma unroll
  for (int e2 = 0; e2 < D / 32; ++e2) {
    bf16x8 even, odd;
    __builtin_amdgcn_sched_barrier(0);
    values.v_pair(e2, even, odd);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      st.o[t][2 * e2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pf[t], st.o[t][2 * e2], 0, 0, 0);
      st.o[t][2 * e2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pf[t], st.o[t][2 * e2 + 1], 0, 0, 0);
    }
  }
}

// ---------------------------------------------------------------------------------------------- kernel

// A partial slot: sums in the order in which lanes hold them, [row tile][four channel tiles][entry][lane] quads of channels (a store
// instruction writes a kilobyte in a row), behind them the rows' shifts and sums.
template <int D>
__device__ __forceinline__ int64_t slot_floats(int rows) { return (int64_t)rows * (D + 2); }
template <int D>
__device__ __forceinline__ int quad_at(int tile, int quad, int entry, int lane) { return (((tile * (D / 64) + quad) * 4 + entry) * 64 + lane) * 4; }

// WIDE: a page holds a block's 32 keys (pages of 16 keys: a block's halves lie on two).
template <int QT, int D, bool WIDE>
__global__ __launch_bounds__(64 * paged_waves(QT, D), paged_waves(QT, D) * paged_resident(QT, D) / 4) void tree_attn_paged_kernel(const PagedParams) {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int KS = D / 32, DT = D / 16, ROWS = 16 * QT, WAVES = paged_waves(QT, D);
  __shared__ f32x4 merge_o[WAVES][QT * DT][64];
  __shared__ float2 merge_ml[WAVES][QT][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Cutter cutter(p, threadIdx.x & 63);
  // (the grid is a multiple of eight)
  const int share = (cutter.places + 7) >> 3, die = blockIdx.x & 7, step = gridDim.x >> 3;
  for (int nth = blockIdx.x >> 3; nth < share; nth += step) {
  const int place_at = die * share + nth;
  if (place_at >= cutter.places) break;
  if (nth >= step) __syncthreads();   // the merge buffers are used again
  const int lane = (int)here(threadIdx.x & 63), col = lane & 15, g4 = lane >> 4;   // (what is made of them is made for every piece)
  const Piece piece = cutter.piece(place_at);
  const int b = piece.b, g = piece.g, y = piece.y, L = piece.len, n = piece.n;
  const int WS = 1 << p->ws_shift, KW = WAVES >> p->ws_shift;   // row slabs, wavefronts that split a slab's keys
  const int slab = wave & (WS - 1), kp = wave >> p->ws_shift;
  const int row0 = y * p->rows_per_group + slab * ROWS;
  if (piece.begin == 0 && threadIdx.x == 0) p->cuts[(b * p->groups + y) * p->Hkv + g] = make_int2(piece.index, piece.count > 1 ? piece.count : 0);

  struct RowInfo { bool exists, valid; int node; int64_t out; };
  auto row_info = [&](int t) {
    RowInfo ri;
    const int rr = row0 + 16 * t + col;
    ri.node = (int)div_rcp((unsigned)rr, (unsigned)p->G, p->g_rcp);
    ri.exists = rr < p->N * p->G;
    ri.valid = ri.exists && ri.node < n;
    ri.out = ((int64_t)b * p->N + ri.node) * p->Hq + g * p->G + (rr - ri.node * p->G);
    return ri;
  };

  RowState<QT, D> st;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    st.m[t] = kNoShift;
    st.l[t] = 0.f;
#pragma unroll
    for (int e = 0; e < DT; ++e) st.o[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int tree_blocks = (n + kBlockKeys - 1) / kBlockKeys;   // the first blocks of a unit
  int blk = piece.begin + kp;                                  // neighbouring wavefronts take neighbouring blocks
  if (row0 < n * p->G && blk < piece.end) {
    // ---- the prefix's blocks in the pages: a half block's bases are scalars, a lane adds its own places
    // (V's codes of D = 64 lie in groups of eight keys: half a piece each; the products' channels of D = 64 are K's, twice)
    const int P = 1 << p->page_shift, codes = page_code_bytes(D, P), scales = page_scale_bytes(D, P), k_block = g4 & (D / 32 - 1);
    const unsigned k_off = (unsigned)(col * (D / 2) + k_block * 16);
    const unsigned v_off = (unsigned)(codes + (D == 128 ? g4 * 256 + col * 16 : (g4 >> 1) * 256 + col * 16 + (g4 & 1) * 8));
    const unsigned ks_off = (unsigned)(2 * codes + k_block * P + col);
    const unsigned vs_off = (unsigned)(2 * codes + scales + (col * (D / 16) / 32) * P + 4 * g4);
    GlobalBytes const pool = (GlobalBytes)p->pages + (int64_t)g * page_head_bytes(D, P);
    ScalarI32 const table = (ScalarI32)p->table + (int64_t)b * p->table_stride;
    const uint32_t page_stride = p->page_stride;
    const int page_shift = p->page_shift, n_pages = p->n_pages;
    constexpr int HALVES = WIDE ? 1 : 2, KEYS = 32 / HALVES;
    struct Ids { int id[HALVES]; };
    auto ids_of = [&](int at) {   // (places of the prefix: block `at` has keys 32 at ..)
      const unsigned t0 = (unsigned)at * kBlockKeys;
      Ids r;
      r.id[0] = table[t0 >> page_shift];
      if constexpr (!WIDE) r.id[1] = table[min(t0 + 16, (unsigned)L - 1) >> page_shift];
      return r;
    };
    auto vis_of = [&](int at, const Ids& ids) {   // bit t: key t is there; block `at` has one at least
      unsigned vis = ~0u >> (32 - min(L - at * kBlockKeys, 32));
#pragma unroll
      for (int half = 0; half < HALVES; ++half)
        if ((unsigned)ids.id[half] >= (unsigned)n_pages) vis &= WIDE ? 0u : half == 0 ? 0xffff0000u : 0x0000ffffu;
      return vis;
    };
    struct Block { GlobalBytes code[HALVES], scale[HALVES]; };
    auto place = [&](int at, const Ids& ids) {
      Block r;
#pragma unroll
      for (int half = 0; half < HALVES; ++half) {
        const unsigned id = (unsigned)ids.id[half] < (unsigned)n_pages ? (unsigned)ids.id[half] : 0u;
        const unsigned in_page = ((unsigned)at * kBlockKeys + 16u * half) & (unsigned)(P - 1);
        GlobalBytes const page = pool + (uint64_t)id * page_stride;
        r.code[half] = page + in_page * (D / 2);
        r.scale[half] = page + in_page;
      }
      return r;
    };
    // (the second 16 keys of a wide block are 16 rows further on)
    auto load_k = [&](PagedK& x, const Block& block) {
      const unsigned k_at = here(k_off), ks_at = here(ks_off);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int half = WIDE ? 0 : kt, further = WIDE ? 16 * kt : 0;
        x.c[kt] = *(const __attribute__((address_space(1))) u32x4*)(block.code[half] + k_at + further * (D / 2));
        x.scale[kt] = ((const __attribute__((address_space(1))) Unaligned*)(block.scale[half] + ks_at + further))->word;   // (the products take its first byte)
      }
    };
    auto load_v = [&](PagedV<D>& x, const Block& block) {
      const unsigned v_at = here(v_off), vs_at = here(vs_off);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int half = WIDE ? 0 : h, further = WIDE ? 16 * h : 0;
        if constexpr (D == 128) {
          const u32x4 w = *(const __attribute__((address_space(1))) u32x4*)(block.code[half] + v_at + further * (D / 2));
#pragma unroll
          for (int i = 0; i < 4; ++i) x.c[4 * h + i] = w[i];
        } else {
          const u32x2 w = *(const __attribute__((address_space(1))) u32x2*)(block.code[half] + v_at + further * (D / 2));
          x.c[2 * h] = w[0]; x.c[2 * h + 1] = w[1];
        }
        x.scale[h] = *(const __attribute__((address_space(1))) unsigned*)(block.scale[half] + vs_at + further);
      }
    };

    // the wavefront's places of the prefix: at, at + KW, .. last
    int at = blk;
    while (at < tree_blocks) at += KW;
    at -= tree_blocks;
    const int end = piece.end - tree_blocks;
    const bool any_prefix = at < end;
    const int last = any_prefix ? at + (end - 1 - at) / KW * KW : 0;
    PagedK keys{}, k_other;
    PagedV<D> v_this{}, v_other;
    Ids ids_next{};
    Block block{};
    unsigned vis_next = 0;
    if (any_prefix) {
      const Ids ids = ids_of(at);
      ids_next = ids_of(min(at + KW, last));
      block = place(at, ids);
      vis_next = vis_of(at, ids);
      load_k(keys, block);
    }
    // the rows' channels that this lane holds, eight at a time: 16 g4 and 16 g4 + 8, and the same 64 further on
    auto channel = [&](int i) { return (i >> 1) * 64 + 16 * g4 + 8 * (i & 1); };
    u32x4 q_row[QT][KS];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const RowInfo ri = row_info(t);
#pragma unroll
      for (int i = 0; i < KS; ++i)
        q_row[t][i] = ri.valid ? *reinterpret_cast<const u32x4*>(p->q + (ri.out * D + channel(i)) * 2) : u32x4{0u, 0u, 0u, 0u};
    }

    bf16x8 pf[QT];
    // ---- blocks of the tree
    for (; blk < min(tree_blocks, piece.end); blk += KW) {
      const int t0 = blk * kBlockKeys;
      const int64_t row = (int64_t)p->Hkv * D * 2;
      const char* kr = p->k_tree + ((int64_t)b * p->N * p->Hkv + g) * (D * 2);
      const char* vr = p->v_tree + ((int64_t)b * p->N * p->Hkv + g) * (D * 2);
      bf16x8 kf[2][KS];
      TreeV<D> values;
      uint64_t tree_mask[QT];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int node = min(t0 + 16 * kt + col, n - 1);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[kt][ks] = *reinterpret_cast<const bf16x8*>(kr + node * row + 2 * channel(ks));
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const RowInfo ri = row_info(t);
        tree_mask[t] = ri.valid ? p->mask[b * p->N + ri.node] : 0ull;
      }
      unsigned wild = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int node = min(t0 + 4 * g4 + key_of(j), n - 1);
        const char* src = vr + node * row + (D / 8) * col;
        if constexpr (D == 128) {
          const u32x4 v4 = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
          for (int i = 0; i < 4; ++i) values.v[j][i] = v4[i];
        } else {
          const u32x2 v2 = *reinterpret_cast<const u32x2*>(src);
          values.v[j][0] = v2[0]; values.v[j][1] = v2[1];
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) wild |= has_wild(values.v[j][i]);
      }
      // A weight of zero does not keep NaN and infinity out of a product. Where the tree's values hold any, they are taken out
      // here and added below to the rows that see them.
      const bool any_wild = __any(wild != 0);
      if (__builtin_expect(any_wild, 0)) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < D / 32; ++i) values.v[j][i] &= ~wild_halves(values.v[j][i]);
      }
      const unsigned there = n - t0 >= kBlockKeys ? ~0u : (1u << (n - t0)) - 1u;
      auto visible = [&](int t) { return (unsigned)(tree_mask[t] >> t0) & there; };
      Scores<QT> s;
      float x[QT][8];
      auto score = [&](Scores<QT>& s) {
        score_tree<QT, D>(s, kf, q_row);
        hide<QT>(s, visible, p->c, g4);
      };
      score(s);
      settle<QT, D>(st, x, exponents<QT, D>(st, s, x, p->c), p->c, score);
      weigh<QT>(x, pf);
      accumulate<QT, D>(st, pf, values);
      if (__builtin_expect(any_wild, 0)) {
#pragma unroll 1
        for (int key = 0; key < kBlockKeys; ++key) {
          if (!((there >> key) & 1u)) break;
          const char* src = vr + (t0 + key) * row;
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            float own = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) own = (key & 3) + 4 * (key >> 4) == j ? (float)pf[t][j] : own;
            const float weight = __shfl(own, 16 * ((key >> 2) & 3) + col);
            if (!((visible(t) >> key) & 1u)) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e2 = 0; e2 < DT / 2; ++e2) {
                const unsigned w2 = *reinterpret_cast<const unsigned*>(src + 2 * (DT * (4 * g4 + i) + 2 * e2));
                const unsigned odd = wild_halves(w2);
                if (odd & 0xffffu) st.o[t][2 * e2][i] += weight * __builtin_bit_cast(float, w2 << 16);
                if (odd >> 16) st.o[t][2 * e2 + 1][i] += weight * __builtin_bit_cast(float, w2 & 0xffff0000u);
              }
          }
        }
      }
    }

    // ---- blocks of the prefix. A turn forms the weights and sums of one block and the scores of the next: its products do not wait
    // for the exponentials, nor these for them. Its values and the keys of the block after it were asked for a turn ahead. The first turn
    // has no block yet (weights of zero: the scores' code stands once), the last one forms its own scores again, for nobody.
    if (any_prefix) {
      SplitQ<D> q[QT];
      float x[QT][8];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        q[t].split(q_row[t], g4);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[t][j] = -INFINITY;
      }
      const float c = p->c;
      unsigned vis_this = 0;   // (no key is there)
      int third = min(at + KW, last);
      at -= KW;
      // (two turns stand in the loop, each with registers of its own for what it asks for: copied from one set to another, loads would be
      // waited for in the turn that asks for them)
      auto turn_of_stream = [&](PagedK& k_this, PagedK& k_third, PagedV<D>& v_this, PagedV<D>& v_next) {
        load_v(v_next, block);
        const unsigned vis = vis_next;
        block = place(third, ids_next);
        vis_next = vis_of(third, ids_next);
        load_k(k_third, block);
        third = min(third + KW, last);
        ids_next = ids_of(third);
        weigh<QT>(x, pf);
        __builtin_amdgcn_sched_barrier(0);
        Scores<QT> s;
        score_block<QT, D>(s, k_this, q);
        __builtin_amdgcn_sched_barrier(0);
        v_this.ready(vis_this, g4);
        accumulate<QT, D>(st, pf, v_this);
        float most;
        if (__builtin_expect(vis != ~0u, 0)) {
          hide<QT>(s, [&](int) { return vis; }, c, g4);
          most = exponents<QT, D>(st, s, x, c);
        } else {
          most = exponents<QT, D>(st, s, x, c);
        }
        settle<QT, D>(st, x, most, c, [&](Scores<QT>& again) {
          score_block<QT, D>(again, k_this, q);
          if (vis != ~0u) hide<QT>(again, [&](int) { return vis; }, c, g4);
        });
        vis_this = vis;
        at += KW;
        return at <= last;
      };
      while (turn_of_stream(keys, k_other, v_this, v_other) && turn_of_stream(k_other, keys, v_other, v_this)) {}
    }
  }
  p = fresh(p);

  // ---- the key-splitting wavefronts of a slab meet in LDS; each writes its share of the (row tile, four channel tiles) quads
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    merge_ml[wave][t][lane] = make_float2(st.m[t], st.l[t]);
#pragma unroll
    for (int e = 0; e < DT; ++e) merge_o[wave][t * DT + e][lane] = st.o[t][e];
  }
  __syncthreads();
  constexpr int kQuads = DT / 4;
  for (int q = kp; q < QT * kQuads; q += KW) {
    const int t = q / kQuads, e0 = 4 * (q - t * kQuads);
    float mm = kNoShift;
    for (int k = 0; k < KW; ++k) mm = fmaxf(mm, merge_ml[slab + k * WS][t][lane].x);
    float l_row = 0.f;
    f32x4 o4[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) o4[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < KW; ++k) {   // in wavefront order: the same bits every time
      const float2 ml = merge_ml[slab + k * WS][t][lane];
      const float a = __builtin_amdgcn_exp2f(ml.x - mm);
      l_row += ml.y * a;
#pragma unroll
      for (int j = 0; j < 4; ++j) o4[j] += merge_o[slab + k * WS][t * DT + e0 + j][lane] * a;
    }
    const RowInfo ri = row_info(t);
    if (!ri.exists) continue;
    if (piece.count == 1) {
      const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t out_at = ri.out * D + DT * (4 * g4 + i) + e0;
        f32x4 val;
#pragma unroll
        for (int j = 0; j < 4; ++j) val[j] = ri.valid ? o4[j][i] * inv : 0.f;
        if (p->out_bf16) {
          bf16x4 pk;
#pragma unroll
          for (int j = 0; j < 4; ++j) pk[j] = (__bf16)val[j];
          *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p->out) + out_at) = pk;
        } else {
          *reinterpret_cast<f32x4*>(static_cast<float*>(p->out) + out_at) = val;
        }
      }
    } else {
      float* part = p->part + piece.index * slot_floats<D>(p->rows_per_group);
      const int tile = slab * QT + t;
      if (g4 == 0 && e0 == 0) *reinterpret_cast<float2*>(part + (int64_t)p->rows_per_group * D + 2 * (16 * tile + col)) = make_float2(mm, l_row);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(part + quad_at<D>(tile, e0 / 4, i, lane)) = f32x4{o4[0][i], o4[1][i], o4[2][i], o4[3][i]};
    }
  }
  }
}

// Joins the pieces of the units that were cut: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s. A wavefront has one entry of a quad
// for sixteen rows, as the pieces' wavefronts left it: four channels of a row a lane.
template <int D>
__global__ __launch_bounds__(256) void tree_attn_paged_join_kernel(const PagedParams p) {
  const int g = blockIdx.y, y = blockIdx.z % p.groups, b = blockIdx.z / p.groups;
  const int2 cut = p.cuts[(b * p.groups + y) * p.Hkv + g];
  if (cut.y == 0) return;
  const int lane = threadIdx.x & 63, item = blockIdx.x * 4 + (threadIdx.x >> 6);   // (row tile, quad, entry)
  const int i = item & 3, quad = (item >> 2) % (D / 64), tile = (item >> 2) / (D / 64);
  const int lr = 16 * tile + (lane & 15), rr = y * p.rows_per_group + lr;
  if (lr >= p.rows_per_group || rr >= p.N * p.G) return;
  const int node = (int)div_rcp((unsigned)rr, (unsigned)p.G, p.g_rcp);
  const int n = min(max(p.n_nodes[b], 0), p.N);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (node < n) {
    const int64_t slot = slot_floats<D>(p.rows_per_group);
    const float* base = p.part + cut.x * slot;
    const float* o_at = base + quad_at<D>(tile, quad, i, lane);
    const float* ml_at = base + (int64_t)p.rows_per_group * D + 2 * lr;
    float M = kNoShift, sum = 0.f;
    for (int s0 = 0; s0 < cut.y; s0 += 8) {   // in order: the same bits every time
      float2 ml[8];
      f32x4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t at = min(s0 + k, cut.y - 1) * slot;
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
        if (s0 + k >= cut.y) break;
        const float wgt = __builtin_amdgcn_exp2f(ml[k].x - M);
        sum += wgt * ml[k].y;
        acc += wgt * o[k];
      }
    }
    acc *= sum == 0.f ? 0.f : 1.0f / sum;
  }
  const int64_t at = (((int64_t)b * p.N + node) * p.Hq + g * p.G + (rr - node * p.G)) * D + (D / 16) * (4 * (lane >> 4) + i) + 4 * quad;
  if (p.out_bf16) {
    bf16x4 pk;
#pragma unroll
    for (int e = 0; e < 4; ++e) pk[e] = (__bf16)acc[e];
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + at) = pk;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = acc;
  }
}

template <int D, bool WIDE>
void launch(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  // a multiple of eight: workgroup w takes places w / 8, one grid's eighth further, .. of die w % 8's share
  const int wgs = pl.max_pieces < pl.resident ? pl.max_pieces : pl.resident;
  const dim3 grid((unsigned)((wgs + 7) / 8 * 8));
  if (pl.QT == 1) hipLaunchKernelGGL((tree_attn_paged_kernel<1, D, WIDE>), grid, dim3(64 * paged_waves(1, D)), 0, stream, p);
  else if (pl.QT == 2) hipLaunchKernelGGL((tree_attn_paged_kernel<2, D, WIDE>), grid, dim3(64 * paged_waves(2, D)), 0, stream, p);
  else if constexpr (D == 64) hipLaunchKernelGGL((tree_attn_paged_kernel<4, D, WIDE>), grid, dim3(64 * paged_waves(4, D)), 0, stream, p);
  if (!pl.may_cut) return;
  const int rows = pl.rows_per_group < p.N * p.G ? pl.rows_per_group : p.N * p.G;
  hipLaunchKernelGGL((tree_attn_paged_join_kernel<D>), dim3((unsigned)((rows + 15) / 16 * (D / 64)), (unsigned)p.Hkv, (unsigned)(p.B * pl.groups)),
                     dim3(256), 0, stream, p);
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
  p.pages = static_cast<const char*>(pages); p.table = block_table; p.kv_len = kv_len; p.n_nodes = n_nodes; p.mask = anc_mask;
  p.out = out; p.cuts = static_cast<int2*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.cuts_bytes);
  p.page_stride = (uint32_t)d.page_stride; p.table_stride = d.table_stride;
  p.B = d.batch; p.N = d.n_nodes_max; p.Hq = d.n_q_heads; p.Hkv = d.n_kv_heads; p.G = d.n_q_heads / d.n_kv_heads;
  p.page_shift = log2_of(d.page_tokens); p.n_pages = d.n_pages; p.max_kv_len = d.max_kv_len;
  p.g_rcp = reciprocal(p.G);
  p.ws_shift = log2_of(pl.WS); p.rows_shift = log2_of(pl.rows_per_group); p.rows_per_group = pl.rows_per_group; p.groups = pl.groups;
  p.max_pieces = pl.max_pieces; p.resident = pl.resident; p.least_blocks = pl.least_blocks; p.whole_blocks = pl.whole_blocks; p.piece_cost = pl.piece_cost; p.forced = d.workgroups;
  p.out_bf16 = d.out_dtype == FSPAD_BF16;
  p.c = c;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const bool wide = d.page_tokens >= kBlockKeys;
  if (d.head_dim == 128) wide ? launch<128, true>(pl, p, stream) : launch<128, false>(pl, p, stream);
  else wide ? launch<64, true>(pl, p, stream) : launch<64, false>(pl, p, stream);
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}
