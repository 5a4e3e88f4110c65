// Tree-masked attention over a paged 4-bit cache (arXiv 2408.15562, Preliminaries, validation phase, as fspad_attn.hip; the
// cache format is in include/fspad.h). gfx950 (CDNA4) only.
//
// One pass over the keys with a running shift and sum per query row. A wavefront owns up to 64 query rows (16-row tiles) of one
// kv head and takes 32-key blocks of K and V from the pages straight into registers, 4 bits an entry; they become bf16 on the
// way into the matrix cores (v_cvt_scalef32_pk_bf16_fp4: two entries and their block's scale in one instruction, exact). The
// layout of the pages is that of the operands:
//   S^T = K Q^T    lane (col, g4), col = lane % 16, g4 = lane / 16, of a 16-key tile kt holds D/4 channels of key 8 (col / 4) +
//                  4 kt + col % 4: one piece of its row, in one block of 32 channels
//   O^T += V^T P^T lane (col, g4) holds D/16 channels of the keys 8 g4 .. 8 g4 + 7, the ones whose scores S^T leaves in it
// so that the weights never leave the lane they arise in. Of a block of V the lane's 8 x D/16 entries turn from key order to
// channel order two bytes at a time (v_perm_b32).
//
// How a call is cut is decided on the device, from lengths it alone knows: the 32-key blocks of all (sequence, kv head, row
// group) units form one list, which the workgroups share evenly. A unit that is one workgroup's goes straight to `out`; of the others
// every piece leaves its un-normalised sums in the workspace and a second kernel joins them.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"
#include "paged_plan.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
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
  float* part;      // partial slots
  int64_t page_stride, table_stride;
  int32_t B, N, Hq, Hkv, G, page_shift, n_pages, max_kv_len;
  int32_t ws_shift, rows_per_group, groups, n_wgs, min_blocks, out_bf16;
  float c;          // softmax scale * log2(e)
};

// The shift of a row moves only when a score exceeds it by more than this (log2 units): weights stay below 2^8, which fp32 sums
// and bf16 weights hold without loss, and accumulators are rescaled almost never after the first blocks.
constexpr float kLazyLog2 = 8.0f;
constexpr float kNoShift = -FLT_MAX;   // below every score: the first visible one moves it

// ------------------------------------------------------------------------------------------------ plan

// What a sequence is made of: `live` row groups of nb blocks each per kv head, the others one entry each (they write zeros).
struct SeqShape {
  int len, n, live, nb;
  unsigned flat;
};
__device__ __forceinline__ SeqShape shape_of(const PagedParams& p, int len, int n) {
  SeqShape s;
  s.len = min(max(len, 0), p.max_kv_len);
  s.n = min(max(n, 0), p.N);
  s.live = (s.n * p.G + p.rows_per_group - 1) / p.rows_per_group;
  s.nb = (s.len + kBlockKeys - 1) / kBlockKeys + (s.n + kBlockKeys - 1) / kBlockKeys;
  s.flat = (unsigned)p.Hkv * (unsigned)(s.live * s.nb + p.groups - s.live);
  return s;
}

// 64 sequences at a time, one a lane, with their first places in the list.
struct SeqChunk {
  int chunk;
  unsigned first, end;   // the lane's first place; the chunk's end
  SeqShape s;
};
__device__ __forceinline__ SeqChunk load_chunk(const PagedParams& p, int chunk, unsigned begin, int lane) {
  SeqChunk c;
  c.chunk = chunk;
  const int b = 64 * chunk + lane;
  c.s = shape_of(p, b < p.B ? p.kv_len[b] : 0, b < p.B ? p.n_nodes[b] : 0);
  if (b >= p.B) c.s.flat = 0;
  const unsigned sum = (unsigned)wave_sum_upto((int)c.s.flat);
  c.first = begin + sum - c.s.flat;
  c.end = begin + (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
  return c;
}

// The even split of T places over W workgroups: the first T % W of them have one more.
struct Split {
  unsigned quot, rem;
  __device__ __forceinline__ unsigned begin(unsigned w) const { return w * quot + min(w, rem); }
  __device__ __forceinline__ unsigned owner(unsigned x) const {
    const unsigned big = rem * (quot + 1);
    return x < big ? x / (quot + 1) : rem + (x - big) / quot;
  }
};

// -------------------------------------------------------------------------------------------- operands

template <int QT, int D>
struct RowState {
  static constexpr int DT = D / 16;
  f32x4 o[QT][DT];   // O^T: lane (col, g4), entry i <-> row 16 t + col, channel DT (4 g4 + i) + e
  float m[QT];       // shift in use (log2 units): within kLazyLog2 of the running maximum
  f32x4 l[QT];       // sum of the rounded weights, formed on the matrix cores (all entries equal)
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

// K and V of a 32-key block of the prefix as they lie in the pages. Keys that are not there (past the length, on a bad page) are
// masked by their scores; their values only have to be finite, which codes are under any scale but 255.
template <int D>
struct PagedK {
  unsigned c[2][D / 32], scale[2];

  __device__ __forceinline__ bf16x8 k_frag(int kt, int ks) const {
    const float f = __builtin_bit_cast(float, scale[kt] << 23);
    const unsigned w = c[kt][ks];
    const u32x4 x = {two_values<0>(w, f), two_values<1>(w, f), two_values<2>(w, f), two_values<3>(w, f)};
    return __builtin_bit_cast(bf16x8, x);
  }
};
template <int D>
struct PagedV {
  unsigned c[D / 16];
  unsigned scale[2];
  float f[8];   // scales of the lane's keys

  __device__ __forceinline__ void ready(unsigned vis, int g4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __builtin_bit_cast(float, ((scale[j >> 2] >> (8 * (j & 3))) & 0xffu) << 23);
    if (vis != ~0u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = ((vis >> (8 * g4 + j)) & 1u) ? f[j] : 1.0f;
    }
  }
  __device__ __forceinline__ void v_pair(int e2, bf16x8& even, bf16x8& odd) const {
    unsigned x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = D == 128 ? two_values(c[j], f[j], e2) : two_values(c[j >> 1], f[j], 2 * (j & 1) + e2);
    turn(x, even, odd);
  }
};

// A block of the tree's own keys, bf16 (rows past the tree's end repeat its last one and are masked).
template <int D>
struct TreeBlock {
  bf16x8 k[2][D / 32];
  unsigned v[8][D / 32];

  __device__ __forceinline__ bf16x8 k_frag(int kt, int ks) const { return k[kt][ks]; }
  __device__ __forceinline__ void v_pair(int e2, bf16x8& even, bf16x8& odd) const {
    unsigned x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[j][e2];
    turn(x, even, odd);
  }
};

__device__ __forceinline__ unsigned wild_halves(unsigned w) {   // all bits of a half that holds NaN or infinity
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

template <int QT>
using Scores = f32x4[QT][2];   // lane (col, g4), [t][kt][i]: key 8 g4 + 4 kt + i against row 16 t + col

template <int QT, int D, typename Keys>
__device__ __forceinline__ void score_block(Scores<QT>& s, const Keys& keys, const bf16x8 (&qf)[QT][D / 32]) {
#pragma unroll
  for (int t = 0; t < QT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const bf16x8 a = keys.k_frag(kt, ks);
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][ks], s[t][kt], 0, 0, 0);
    }
}

// Hides what a row does not see; visible(t): the 32 keys that this lane's row of tile t does.
template <int QT, typename VisibleFn>
__device__ __forceinline__ void hide(Scores<QT>& s, VisibleFn&& visible, float c, int g4) {
  const float hidden = c < 0.f ? INFINITY : -INFINITY;   // (times c: below every score)
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const unsigned vis = visible(t) >> (8 * g4);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[t][j >> 2][j & 3] = ((vis >> j) & 1u) ? s[t][j >> 2][j & 3] : hidden;
  }
}

// Exponents of the weights, under the shifts in use or, where a score is too far above its row's, under shifts that move.
template <int QT, int D>
__device__ __forceinline__ void exponents(RowState<QT, D>& st, const Scores<QT>& s, float (&x)[QT][8], float c) {
  bool grow = false;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float m = st.m[t];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[t][j] = fmaf(s[t][j >> 2][j & 3], c, -m);
    const float top = fmaxf(fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3])), fmaxf(fmaxf(x[t][4], x[t][5]), fmaxf(x[t][6], x[t][7])));
    grow = grow || top > kLazyLog2;
  }
  if (__any(grow)) {   // rare: the rows' shifts move to their running maxima
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
}

// Weights are rounded to bf16, which is what the matrix cores take; their sum is that of the rounded ones.
template <int QT, int D, typename Values>
__device__ __forceinline__ void accumulate(RowState<QT, D>& st, const float (&x)[QT][8], const Values& values, bf16x8 (&pf)[QT]) {
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) pf[t][j] = (__bf16)__builtin_amdgcn_exp2f(x[t][j]);
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
#pragma unroll
  for (int t = 0; t < QT; ++t) st.l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t], st.l[t], 0, 0, 0);
#pragma unroll
  for (int e2 = 0; e2 < D / 32; ++e2) {
    bf16x8 even, odd;
    values.v_pair(e2, even, odd);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      st.o[t][2 * e2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pf[t], st.o[t][2 * e2], 0, 0, 0);
      st.o[t][2 * e2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pf[t], st.o[t][2 * e2 + 1], 0, 0, 0);
    }
  }
}

// ---------------------------------------------------------------------------------------------- kernel

template <int QT, int D>
__global__ __launch_bounds__(256, QT <= 2 ? 2 : 1) void tree_attn_paged_kernel(const PagedParams p) {
  constexpr int KS = D / 32, DT = D / 16, ROWS = 16 * QT;
  __shared__ f32x4 merge_o[4][QT * DT][64];
  __shared__ float2 merge_ml[4][QT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  const int WS = 1 << p.ws_shift, KW = 4 >> p.ws_shift;   // row slabs, wavefronts that split a slab's keys
  const int slab = wave & (WS - 1), kp = wave >> p.ws_shift;
  const int P = 1 << p.page_shift;
  // this lane's places in a block's codes and scales (pages of 16 keys: the block's second half is at the start of another page)
  const bool k_late = col >= 8, v_late = g4 >= 2;
  const int k_key = 8 * (col >> 2) + (col & 3) - (P == 16 && k_late ? 16 : 0), v_key = 8 * g4 - (P == 16 && v_late ? 16 : 0);
  const unsigned k_off = (unsigned)(k_key * (D / 2) + g4 * (D / 8)), ks_off = (unsigned)((g4 * (D / 4) / 32) * P + k_key);
  const unsigned v_off = (unsigned)(v_key * (D / 2) + col * 16), vs_off = (unsigned)((col * (D / 16) / 32) * P + v_key);
  const int head_bytes = page_head_bytes(D, P), codes = page_code_bytes(D, P), scales = page_scale_bytes(D, P);

  // this workgroup's places of the list
  SeqChunk ch = load_chunk(p, 0, 0, lane);
  unsigned total = ch.end;
  if (p.B > 64) {
    for (int c = 1; 64 * c < p.B; ++c) total = load_chunk(p, c, total, lane).end;
  }
  const unsigned wgs = min((unsigned)p.n_wgs, max(total / (unsigned)p.min_blocks, 1u));
  const unsigned w = blockIdx.x;
  if (w >= wgs) return;
  Split split;
  split.quot = total / wgs;
  split.rem = total - split.quot * wgs;
  unsigned r = split.begin(w);
  const unsigned r_end = split.begin(w + 1);

  while (r < r_end) {
    while (r >= ch.end) ch = load_chunk(p, ch.chunk + 1, ch.end, lane);   // (r lies before the list's end)
    const int in_chunk = 63 - __builtin_clzll(__ballot(ch.first <= r && ch.s.flat > 0));
    const int b = 64 * ch.chunk + in_chunk;
    const int L = __builtin_amdgcn_readlane(ch.s.len, in_chunk), n = __builtin_amdgcn_readlane(ch.s.n, in_chunk);
    const int nb = __builtin_amdgcn_readlane(ch.s.nb, in_chunk), live = __builtin_amdgcn_readlane(ch.s.live, in_chunk);
    const unsigned rel = r - (unsigned)__builtin_amdgcn_readlane((int)ch.first, in_chunk);
    const unsigned live_places = (unsigned)(p.Hkv * live) * (unsigned)nb;
    const bool dead = rel >= live_places;   // a row group without nodes
    int u, seg_begin, g, y;
    if (dead) {
      const int others = p.groups - live, x = (int)(rel - live_places);
      u = p.Hkv * live + x;
      g = x / others;
      y = live + (x - g * others);
      seg_begin = 0;
    } else {
      u = (int)(rel / (unsigned)nb);
      seg_begin = (int)(rel - (unsigned)u * (unsigned)nb);
      g = u / live;
      y = u - g * live;
    }
    const int n_blocks = dead ? 1 : nb;
    const int seg_count = min(n_blocks - seg_begin, (int)(r_end - r));
    const bool whole_unit = seg_count == n_blocks;
    const int unit = b * p.Hkv * p.groups + u;   // in the list's order
    if (seg_begin == 0 && threadIdx.x == 0) {
      const int pieces = whole_unit ? 0 : (int)(split.owner(r + (unsigned)n_blocks - 1) - w) + 1;
      p.cuts[(b * p.Hkv + g) * p.groups + y] = make_int2(unit + (int)w, pieces);
    }
    const int row0 = y * p.rows_per_group + slab * ROWS;
    const bool slab_live = !dead && row0 < n * p.G;
    const int tree_blocks = (n + kBlockKeys - 1) / kBlockKeys;   // the first blocks of a unit
    const int blk_end = seg_begin + seg_count;

    struct RowInfo { bool exists, valid; int node; int64_t out; };
    auto row_info = [&](int t) {
      RowInfo ri;
      const int rr = row0 + 16 * t + col;
      ri.node = rr / p.G;
      ri.exists = rr < p.N * p.G;
      ri.valid = ri.exists && ri.node < n;
      ri.out = ((int64_t)b * p.N + ri.node) * p.Hq + g * p.G + (rr - ri.node * p.G);
      return ri;
    };

    // ---- the prefix's blocks in the pages: bases are scalars, a lane adds what it adds to every block
    GlobalBytes const pool = (GlobalBytes)p.pages + (int64_t)g * head_bytes;
    ScalarI32 const table = (ScalarI32)p.table + (int64_t)b * p.table_stride;
    struct Ids { int a, b; };   // pages of the first and the second 16 keys
    auto ids_of = [&](int at) {   // (places of the prefix from here on: block `at` has keys 32 at ..)
      const int t0 = at * kBlockKeys;
      return Ids{table[t0 >> p.page_shift], table[min(t0 + 16, L - 1) >> p.page_shift]};
    };
    auto vis_of = [&](int at, const Ids& ids) {   // bit t: key t is there
      const int left = L - at * kBlockKeys;
      unsigned vis = left >= kBlockKeys ? ~0u : (1u << left) - 1u;
      if ((unsigned)ids.a >= (unsigned)p.n_pages) vis &= 0xffff0000u;
      if ((unsigned)ids.b >= (unsigned)p.n_pages) vis &= 0x0000ffffu;
      return vis;
    };
    auto page_base = [&](int id) { return pool + ((unsigned)id < (unsigned)p.n_pages ? id : 0) * p.page_stride; };
    auto load_k = [&](PagedK<D>& x, int at, const Ids& ids) {
      const int in_page = at * kBlockKeys & (P - 1);
      GlobalBytes code = page_base(ids.a);
      if (P == 16 && k_late) code = page_base(ids.b);
      GlobalBytes scale = code + 2 * codes + in_page;
      code += in_page * (D / 2);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        if constexpr (D == 128) {
          const u32x4 w = *(const __attribute__((address_space(1))) u32x4*)(code + (k_off + kt * 4 * (D / 2)));
#pragma unroll
          for (int i = 0; i < 4; ++i) x.c[kt][i] = w[i];
        } else {
          const u32x2 w = *(const __attribute__((address_space(1))) u32x2*)(code + (k_off + kt * 4 * (D / 2)));
          x.c[kt][0] = w[0]; x.c[kt][1] = w[1];
        }
        x.scale[kt] = *(const __attribute__((address_space(1))) unsigned char*)(scale + (ks_off + 4 * kt));
      }
    };
    auto load_v = [&](PagedV<D>& x, int at, const Ids& ids) {
      const int in_page = at * kBlockKeys & (P - 1);
      GlobalBytes code = page_base(ids.a);
      if (P == 16 && v_late) code = page_base(ids.b);
      GlobalBytes scale = code + 2 * codes + scales + in_page;
      code += codes + in_page * (D / 2);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const u32x4 w = *(const __attribute__((address_space(1))) u32x4*)(code + (v_off + 256 * h));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.c[4 * h + i] = w[i];
      }
      const u32x2 w = *(const __attribute__((address_space(1))) u32x2*)(scale + vs_off);
      x.scale[0] = w[0]; x.scale[1] = w[1];
    };

    int blk = seg_begin + kp;
    const bool active = slab_live && blk < blk_end;
    // the wavefront's places of the prefix: at, at + KW, .. last
    int at = blk;
    while (at < tree_blocks) at += KW;
    at -= tree_blocks;
    const bool any_prefix = slab_live && at + tree_blocks < blk_end;
    const int last = at + (any_prefix ? (blk_end - tree_blocks - 1 - at) / KW * KW : 0);
    PagedK<D> k_now{};
    PagedV<D> v_now{};
    Ids ids_now{0, 0}, ids_next{0, 0}, ids_third{0, 0};
    if (any_prefix) {
      ids_now = ids_of(at);
      load_k(k_now, at, ids_now);
      load_v(v_now, at, ids_now);
      ids_next = ids_of(min(at + KW, last));
    }

    bf16x8 qf[QT][KS];
    uint64_t tree_mask[QT];
    RowState<QT, D> st;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const RowInfo ri = row_info(t);
      const bool valid = ri.valid && active;
      tree_mask[t] = valid ? p.mask[b * p.N + ri.node] : 0ull;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 z;
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = (__bf16)0.f;
        qf[t][ks] = valid ? *reinterpret_cast<const bf16x8*>(p.q + (ri.out * D + (D / 4) * g4 + 8 * ks) * 2) : z;
      }
      st.m[t] = kNoShift;
      st.l[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < DT; ++e) st.o[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    if (active) {
      bf16x8 pf[QT];
      // ---- blocks of the tree
      for (; blk < min(tree_blocks, blk_end); blk += KW) {
        const int t0 = blk * kBlockKeys;
        TreeBlock<D> x;
        const int64_t row = (int64_t)p.Hkv * D * 2;
        const char* kr = p.k_tree + ((int64_t)b * p.N * p.Hkv + g) * (D * 2);
        const char* vr = p.v_tree + ((int64_t)b * p.N * p.Hkv + g) * (D * 2);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const int node = min(t0 + 8 * (col >> 2) + 4 * kt + (col & 3), n - 1);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) x.k[kt][ks] = *reinterpret_cast<const bf16x8*>(kr + node * row + (D / 2) * g4 + 16 * ks);
        }
        unsigned wild = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int node = min(t0 + 8 * g4 + j, n - 1);
          const char* src = vr + node * row + (D / 8) * col;
          if constexpr (D == 128) {
            const u32x4 v4 = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[j][i] = v4[i];
          } else {
            const u32x2 v2 = *reinterpret_cast<const u32x2*>(src);
            x.v[j][0] = v2[0]; x.v[j][1] = v2[1];
          }
#pragma unroll
          for (int i = 0; i < D / 32; ++i) wild |= wild_halves(x.v[j][i]);
        }
        // A weight of zero does not keep NaN and infinity out of a product. Where the tree's values hold any, they are taken out
        // here and added below to the rows that see them.
        const bool any_wild = __any(wild != 0);
        if (any_wild) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) x.v[j][i] &= ~wild_halves(x.v[j][i]);
        }
        const unsigned there = n - t0 >= kBlockKeys ? ~0u : (1u << (n - t0)) - 1u;
        auto visible = [&](int t) { return (unsigned)(tree_mask[t] >> t0) & there; };
        Scores<QT> sc;
        float ex[QT][8];
        score_block<QT, D>(sc, x, qf);
        hide<QT>(sc, visible, p.c, g4);
        exponents<QT, D>(st, sc, ex, p.c);
        accumulate<QT, D>(st, ex, x, pf);
        if (any_wild) {
#pragma unroll 1
          for (int key = 0; key < kBlockKeys; ++key) {
            if (!((there >> key) & 1u)) break;
            const char* src = vr + (t0 + key) * row;
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              float own = 0.f;
#pragma unroll
              for (int j = 0; j < 8; ++j) own = (key & 7) == j ? (float)pf[t][j] : own;
              const float weight = __shfl(own, 16 * (key >> 3) + col);
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
      // ---- blocks of the prefix. The scores of the next block are formed beside the weights and sums of this one: its products do not
      // wait for the exponentials, nor these for them. Behind the last block the last one's are formed again, for nobody.
      if (any_prefix) {
        Scores<QT> s_now;
        score_block<QT, D>(s_now, k_now, qf);
        int next = min(at + KW, last);
        load_k(k_now, next, ids_next);
        for (;;) {
          const unsigned vis = vis_of(at, ids_now);
          const int third = min(next + KW, last);
          ids_third = ids_of(third);
          PagedV<D> v_next;
          load_v(v_next, next, ids_next);
          if (vis != ~0u) hide<QT>(s_now, [&](int) { return vis; }, p.c, g4);
          float x[QT][8];
          exponents<QT, D>(st, s_now, x, p.c);
          v_now.ready(vis, g4);
          Scores<QT> s_next;
          score_block<QT, D>(s_next, k_now, qf);
          load_k(k_now, third, ids_third);
          accumulate<QT, D>(st, x, v_now, pf);
          if (at == last) break;
#pragma unroll
          for (int t = 0; t < QT; ++t) { s_now[t][0] = s_next[t][0]; s_now[t][1] = s_next[t][1]; }
          v_now = v_next;
          at = next; next = third;
          ids_now = ids_next; ids_next = ids_third;
        }
      }
    }

    // ---- the key-splitting wavefronts of a slab meet in LDS; each writes its share of the (row tile, four channel tiles) quads
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      merge_ml[wave][t][lane] = make_float2(st.m[t], st.l[t][0]);
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
      if (whole_unit) {
        const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t at = ri.out * D + DT * (4 * g4 + i) + e0;
          f32x4 val;
#pragma unroll
          for (int j = 0; j < 4; ++j) val[j] = ri.valid ? o4[j][i] * inv : 0.f;
          if (p.out_bf16) {
            bf16x4 pk;
#pragma unroll
            for (int j = 0; j < 4; ++j) pk[j] = (__bf16)val[j];
            *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + at) = pk;
          } else {
            *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = val;
          }
        }
      } else if (ri.valid) {
        float* slot = p.part + (int64_t)(unit + (int)w) * p.rows_per_group * (D + 2);
        const int lr = slab * ROWS + 16 * t + col;
        if (g4 == 0 && e0 == 0) *reinterpret_cast<float2*>(slot + (int64_t)p.rows_per_group * D + 2 * lr) = make_float2(mm, l_row);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(slot + (int64_t)lr * D + DT * (4 * g4 + i) + e0) = f32x4{o4[0][i], o4[1][i], o4[2][i], o4[3][i]};
      }
    }
    r += (unsigned)seg_count;
    if (r < r_end) __syncthreads();   // the merge buffers are used again
  }
}

// Joins the pieces of the units that were cut: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s. A thread has four channels of a row.
template <int D>
__global__ __launch_bounds__(256) void tree_attn_paged_join_kernel(const PagedParams p) {
  const int g = blockIdx.y % p.Hkv, y = blockIdx.y / p.Hkv, b = blockIdx.z;
  const int2 cut = p.cuts[(b * p.Hkv + g) * p.groups + y];
  if (cut.y == 0) return;
  constexpr int TPR = D / 4;
  const int lr = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, d0 = 4 * (threadIdx.x % TPR);
  const int rr = y * p.rows_per_group + lr;
  if (lr >= p.rows_per_group || rr >= p.N * p.G) return;
  const int node = rr / p.G;
  const int n = min(max(p.n_nodes[b], 0), p.N);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (node < n) {
    const int64_t slot_floats = (int64_t)p.rows_per_group * (D + 2);
    const float* base = p.part + cut.x * slot_floats;
    const float* o_at = base + (int64_t)lr * D + d0;
    const float* ml_at = base + (int64_t)p.rows_per_group * D + 2 * lr;
    float M = kNoShift, sum = 0.f;
    for (int s0 = 0; s0 < cut.y; s0 += 4) {   // in order: the same bits every time
      float2 ml[4];
      f32x4 o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t at = min(s0 + k, cut.y - 1) * slot_floats;
        ml[k] = *reinterpret_cast<const float2*>(ml_at + at);
        o[k] = *reinterpret_cast<const f32x4*>(o_at + at);
      }
      float mx = M;
#pragma unroll
      for (int k = 0; k < 4; ++k) mx = fmaxf(mx, ml[k].x);
      const float a = __builtin_amdgcn_exp2f(M - mx);
      acc *= a;
      sum *= a;
      M = mx;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (s0 + k >= cut.y) break;
        const float wgt = __builtin_amdgcn_exp2f(ml[k].x - M);
        sum += wgt * ml[k].y;
        acc += wgt * o[k];
      }
    }
    acc *= sum == 0.f ? 0.f : 1.0f / sum;
  }
  const int64_t at = (((int64_t)b * p.N + node) * p.Hq + g * p.G + (rr - node * p.G)) * D + d0;
  if (p.out_bf16) {
    bf16x4 pk;
#pragma unroll
    for (int e = 0; e < 4; ++e) pk[e] = (__bf16)acc[e];
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + at) = pk;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = acc;
  }
}

template <int D>
void launch(const PagedPlan& pl, const PagedParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)pl.n_wgs);
  switch (pl.QT) {
    case 1: hipLaunchKernelGGL((tree_attn_paged_kernel<1, D>), grid, dim3(256), 0, stream, p); break;
    case 2: hipLaunchKernelGGL((tree_attn_paged_kernel<2, D>), grid, dim3(256), 0, stream, p); break;
    case 3: hipLaunchKernelGGL((tree_attn_paged_kernel<3, D>), grid, dim3(256), 0, stream, p); break;
    default: hipLaunchKernelGGL((tree_attn_paged_kernel<4, D>), grid, dim3(256), 0, stream, p); break;
  }
  constexpr int kRows = 256 / (D / 4);
  const int rows = pl.rows_per_group < p.N * p.G ? pl.rows_per_group : p.N * p.G;
  hipLaunchKernelGGL((tree_attn_paged_join_kernel<D>), dim3((unsigned)((rows + kRows - 1) / kRows), (unsigned)(p.Hkv * pl.groups), (unsigned)p.B),
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
  p.page_stride = d.page_stride; p.table_stride = d.table_stride;
  p.B = d.batch; p.N = d.n_nodes_max; p.Hq = d.n_q_heads; p.Hkv = d.n_kv_heads; p.G = d.n_q_heads / d.n_kv_heads;
  p.page_shift = log2_of(d.page_tokens); p.n_pages = d.n_pages; p.max_kv_len = d.max_kv_len;
  p.ws_shift = log2_of(pl.WS); p.rows_per_group = pl.rows_per_group; p.groups = pl.groups; p.n_wgs = pl.n_wgs; p.min_blocks = pl.min_blocks;
  p.out_bf16 = d.out_dtype == FSPAD_BF16;
  p.c = c;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (d.head_dim == 128) launch<128>(pl, p, stream);
  else launch<64>(pl, p, stream);
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}
