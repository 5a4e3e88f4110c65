// The two forms of a wavefront's work in the attention over a paged 4-bit cache: what its lanes hold of a 32-key block and of its
// query rows, and the products. What an 8-bit cache's blocks change of them is in paged_forms_fp8.h (PLAIN: channels and keys in the order of
// its pages). Internal to the library. gfx950 (CDNA4) only.
//
// Form16: 16 query rows, on 16x16 products (one token of up to 16 heads, small trees). Form32: tiles of 32 rows, on 32x32 ones, which leave
// the other wavefront of a SIMD more room: beside a stream of 16x16x32 bf16 products one of its vector instructions takes 8.5 clocks,
// beside 32x32x16 ones 6.5 (5.3 alone); 8.7 and 7.0 beside the block-scaled ones.
//
// In both forms the weights never leave the lane they arise in: the keys whose scores S^T = K Q^T leaves in a lane are those that
// the lane holds of V for O^T += V^T P^T.
#ifndef FSPAD_PAGED_FORMS_H
#define FSPAD_PAGED_FORMS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_layout.h"
#include "stream_gemm.h"

namespace fspad_detail {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef const __attribute__((address_space(1))) char* GlobalBytes;

// A lane's number, as it stands here: what is made of it is not made ahead of a loop and kept. (An offset that was widened to 64 bits there
// would be added to every address by instructions of its own, instead of by the load.)
__device__ __forceinline__ unsigned here(unsigned offset) {
  asm volatile("" : "+v"(offset));
  return offset;
}

template <typename T>
__device__ __forceinline__ T fetch(GlobalBytes p) { return *(const __attribute__((address_space(1))) T*)p; }

// Two values of a byte of codes, times the scale: the conversion takes the exponent of its scale, what lies around that does not
// matter, and an exponent of all ones makes NaN of every code. (byte: a constant once unrolled)
template <int BYTE>
__device__ __forceinline__ unsigned two_values(unsigned codes, float scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
__device__ __forceinline__ unsigned two_values(unsigned codes, float scale, int byte) {
  return byte == 0 ? two_values<0>(codes, scale) : byte == 1 ? two_values<1>(codes, scale) : byte == 2 ? two_values<2>(codes, scale)
                                                                                           : two_values<3>(codes, scale);
}
__device__ __forceinline__ float bf16_at(unsigned pair, int upper) { return __builtin_bit_cast(float, upper ? pair & 0xffff0000u : pair << 16); }
// byte j of a word of scales, at a float's exponent
__device__ __forceinline__ float scale_of(unsigned word, int j) { return __builtin_bit_cast(float, j == 3 ? word >> 1 : word << (23 - 8 * j)); }

// From (channel, next channel) of two neighbouring keys: the two keys of one channel.
__device__ __forceinline__ unsigned pair_low(unsigned first, unsigned second) { return __builtin_amdgcn_perm(second, first, 0x05040100u); }
__device__ __forceinline__ unsigned pair_high(unsigned first, unsigned second) { return __builtin_amdgcn_perm(second, first, 0x07060302u); }

// NaN or infinity in either half (an exponent of all ones carries into the sign's place when one is added to it), and all bits of such halves.
__device__ __forceinline__ unsigned has_wild(unsigned w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ unsigned wild_halves(unsigned w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Query rows as the block-scaled products take them: row = hi + lo, each fp8 (e4m3, 4 significant bits) times a power of two of the
// row. A bf16 value has 8 significant bits: hi takes the upper four, and what is left of them is a multiple of the value's last
// place, eight at most, which lo holds exactly. With the row's largest magnitude at 128 .. 256 in hi's units (and what is left of it
// below 256 in lo's, 32 times finer) this holds down to 2^-14 of the largest; below that a value is off by 2^-22 of the largest at
// most. Rows with NaN or infinity have the scale that is NaN.
// WORDS: pairs of the row that the lane holds; `top`: the row's largest magnitude, bf16 bits without the sign.
template <int WORDS>
__device__ __forceinline__ void split_row(const unsigned (&x)[WORDS], unsigned top, int (&hi)[WORDS / 2], int (&lo)[WORDS / 2], int& hi_scale, int& lo_scale) {
  const int e = max((int)(top >> 7), 13) - 7;   // hi's scale byte; lo's is 5 less
  const bool wild = top >= 0x7f80u;
  const float to_hi = __builtin_bit_cast(float, (254 - e) << 23);   // 2^(127 - e); e <= 248
#pragma unroll
  for (int i = 0; i < WORDS / 2; ++i) {
    hi[i] = lo[i] = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const unsigned w = x[2 * i + k];
      const float a = wild ? 0.f : __builtin_bit_cast(float, w << 16) * to_hi, b = wild ? 0.f : __builtin_bit_cast(float, w & 0xffff0000u) * to_hi;
      const int h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
      const f32x2 back = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
      const int l = __builtin_amdgcn_cvt_pk_fp8_f32((a - back[0]) * 32.f, (b - back[1]) * 32.f, 0, false);
      hi[i] |= (h & 0xffff) << (16 * k);
      lo[i] |= (l & 0xffff) << (16 * k);
    }
  }
  hi_scale = wild ? 255 : e;
  lo_scale = wild ? 255 : e - 5;
}
template <int WORDS>
__device__ __forceinline__ unsigned top_of(const unsigned (&x)[WORDS]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < WORDS; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
  return top;
}

// Where a block lies: its halves' codes and scales of the kv head, one half where a page holds all of its 32 keys.
template <bool WIDE>
struct BlockPlace {
  static constexpr int HALVES = WIDE ? 1 : 2;
  GlobalBytes code[HALVES], scale[HALVES];
};

// ---------------------------------------------------------------------------------------------------------------------------
// Lane (col, g4) = (lane % 16, lane / 16).
//   S^T: v_mfma_scale_f32_16x16x128_f8f6f4, K's codes and scales as they are: one block of 32 channels of keys col and 16 + col. D = 128 in
//        two products (hi, lo); D = 64 in one, K's 64 channels twice in its 128.
//   O^T: v_mfma_f32_16x16x32_bf16: D/16 channels of keys 4 g4 .. 4 g4 + 3 and 16 more, bf16 by v_cvt_scalef32_pk_bf16_fp4 (V's scales run along
//        the channels, not along the keys that are summed over), turned from key to channel order two bytes at a time.
template <int D, bool PLAIN = false>
struct Form16 {
  static constexpr int HEAD_DIM = D, TILE = 16, RT = 1, ROWS = 16, NX = 8, E = D / 16, KS = D / 32;
  static constexpr int QUADS = D / 16;   // quads of channels of a row that a lane holds

  __device__ static __forceinline__ int row(int lane) { return lane & 15; }
  __device__ static __forceinline__ int first_key(int lane) { return (PLAIN ? 8 : 4) * (lane >> 4); }
  __device__ static constexpr int key_of(int j) { return PLAIN ? j : (j & 3) + 16 * (j >> 2); }   // less the lane's first
  // the key that row m of the products' operand kt is
  __device__ static __forceinline__ int operand_key(int kt, int m) { return PLAIN ? 8 * (m >> 2) + 4 * kt + (m & 3) : 16 * kt + m; }
  __device__ static __forceinline__ float row_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
  }

  struct State {
    f32x4 o[E];   // entry i <-> channel E (4 g4 + i) + e; PLAIN: with KS sums of each half of the channels, KS (16 (e / KS) + 4 g4 + i) + e % KS
    float m[RT], l[RT];
  };
  __device__ static __forceinline__ void clear(State& st, float m) {
    st.m[0] = m;
    st.l[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) st.o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ static __forceinline__ void rescale(State& st, int, float a) {
    st.l[0] *= a;
#pragma unroll
    for (int e = 0; e < E; ++e) st.o[e] *= a;
  }
  __device__ static __forceinline__ float row_sum(const State& st, int) { return st.l[0]; }
  // quad q: four channels from channel(q, lane) on
  __device__ static __forceinline__ f32x4 quad(const State& st, int, int q) {
    if constexpr (PLAIN && D == 64) {   // (two entries' channels follow one another)
      const int i = 2 * (q & 1), e = 2 * (q >> 1);
      return f32x4{st.o[e][i], st.o[e + 1][i], st.o[e][i + 1], st.o[e + 1][i + 1]};
    }
    const int i = q & 3, e = 4 * (q >> 2);
    return f32x4{st.o[e][i], st.o[e + 1][i], st.o[e + 2][i], st.o[e + 3][i]};
  }
  __device__ static __forceinline__ int channel(int q, int lane) {
    if constexpr (PLAIN) return D == 64 ? 2 * (16 * (q >> 1) + 4 * (lane >> 4) + 2 * (q & 1)) : 4 * (16 * (q >> 2) + 4 * (lane >> 4) + (q & 3));
    else return E * (4 * (lane >> 4) + (q & 3)) + 4 * (q >> 2);
  }

  // ---- query rows: 16-byte pieces of a row, as the tree's products take them one by one
  static constexpr int PIECES = D / 32;
  __device__ static __forceinline__ int piece_channel(int i, int lane) { return (i >> 1) * 64 + 16 * (lane >> 4) + 8 * (i & 1); }
  struct Query {
    i32x8 v[RT][D / 64];   // D = 128: hi, lo; D = 64: hi in the first half, lo in the second
    int scale[RT];         // D = 128: hi's in the first byte, lo's in the second
  };
  __device__ static __forceinline__ void split(Query& q, int t, const u32x4 (&piece)[PIECES], int lane) {
    unsigned x[4 * PIECES];
#pragma unroll
    for (int i = 0; i < 4 * PIECES; ++i) x[i] = piece[i >> 2][i & 3];
    unsigned top = top_of(x);
    top = max(top, (unsigned)__shfl_xor((int)top, 16));
    top = max(top, (unsigned)__shfl_xor((int)top, 32));
    int hi[2 * PIECES], lo[2 * PIECES], s_hi, s_lo;
    split_row(x, top, hi, lo, s_hi, s_lo);
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { q.v[t][0][i] = hi[i]; q.v[t][D / 64 - 1][i] = lo[i]; }
      q.scale[t] = s_hi | s_lo << 8;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) { q.v[t][0][i] = hi[i]; q.v[t][0][4 + i] = lo[i]; }
      q.scale[t] = lane < 32 ? s_hi : s_lo;   // (a lane's scale is that of the products' channels 32 g4 .. + 31)
    }
  }

  // ---- blocks of the prefix
  struct Keys {
    u32x4 c[2];
    unsigned scale[2];
  };
  struct Values {
    unsigned c[D / 16], scale[2];
  };
  static constexpr bool HEADS_FIRST = false;   // the order of a call's units
  // where a block's codes and scales start in a head's part of a page, in which a lane's Offsets are counted
  __device__ static constexpr int head_bytes(int P) { return page_head_bytes(D, P); }
  __device__ static __forceinline__ unsigned block_codes(unsigned in_page) { return in_page * (D / 2); }
  __device__ static __forceinline__ unsigned block_scales(unsigned in_page) { return in_page; }
  struct Offsets { unsigned k, ks, v, vs; };
  template <bool WIDE>
  __device__ static __forceinline__ Offsets offsets(int lane, int P) {
    const int col = lane & 15, g4 = lane >> 4, codes = page_code_bytes(D, P), scales = page_scale_bytes(D, P), block = g4 & (D / 32 - 1);
    Offsets o;
    o.k = (unsigned)(col * (D / 2) + block * 16);
    o.ks = (unsigned)(2 * codes + block * P + col);
    // (V's codes of D = 64 lie in groups of eight keys: half a piece each)
    o.v = (unsigned)(codes + (D == 128 ? g4 * 256 + col * 16 : (g4 >> 1) * 256 + col * 16 + (g4 & 1) * 8));
    o.vs = (unsigned)(2 * codes + scales + (col * E / 32) * P + 4 * g4);
    return o;
  }
  template <bool WIDE>
  __device__ static __forceinline__ void load_keys(Keys& x, const BlockPlace<WIDE>& at, const Offsets& off, int, int) {
    const unsigned k = here(off.k), ks = here(off.ks);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {   // (the second 16 keys of a wide block are 16 rows further on)
      const int half = WIDE ? 0 : kt, further = WIDE ? 16 * kt : 0;
      x.c[kt] = fetch<u32x4>(at.code[half] + k + further * (D / 2));
      x.scale[kt] = fetch<uint8_t>(at.scale[half] + ks + further);
    }
  }
  template <bool WIDE>
  __device__ static __forceinline__ void load_values(Values& x, const BlockPlace<WIDE>& at, const Offsets& off, int) {
    const unsigned v = here(off.v), vs = here(off.vs);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int half = WIDE ? 0 : h, further = WIDE ? 16 * h : 0;
      if constexpr (D == 128) {
        const u32x4 w = fetch<u32x4>(at.code[half] + v + further * (D / 2));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.c[4 * h + i] = w[i];
      } else {
        const u32x2 w = fetch<u32x2>(at.code[half] + v + further * (D / 2));
        x.c[2 * h] = w[0]; x.c[2 * h + 1] = w[1];
      }
      x.scale[h] = fetch<unsigned>(at.scale[half] + vs + further);
    }
  }
  // Keys that are not there: their values only have to be finite, which codes are under any scale but 255.
  __device__ static __forceinline__ void mask_values(Values& x, unsigned vis, int lane) {
    const unsigned own = vis >> here(first_key(lane));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!((own >> key_of(j)) & 1u)) x.scale[j >> 2] = (x.scale[j >> 2] & ~(0xffu << (8 * (j & 3)))) | (0x7fu << (8 * (j & 3)));
  }
  __device__ static __forceinline__ void score(float (&s)[RT][NX], const Keys& keys, const Query& q) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const u32x4 c = keys.c[kt];
      const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
      f32x4 r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.v[0][0], f32x4{0.f, 0.f, 0.f, 0.f}, 4 /* a: fp4 */, 0 /* b: e4m3 */, 0,
                                                                 (int)keys.scale[kt], 0, q.scale[0]);
      if constexpr (D == 128)
        r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.v[0][D / 64 - 1], r, 4, 0, 0, (int)keys.scale[kt], 1 /* the second byte */, q.scale[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][4 * kt + i] = r[i];
    }
  }
  __device__ static __forceinline__ void add_weights(State& st, const u32x4 (&w)[RT][1]) {
    bf16x8 ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.0f;
    st.l[0] += __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, w[0][0]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0)[0];   // (all entries equal)
  }
  template <typename PairFn, typename HalfFn>
  __device__ static __forceinline__ void add(State& st, const u32x4 (&w)[RT][1], PairFn&& pairs, HalfFn&& halfway) {
    add_weights(st, w);
#pragma unroll
    for (int e2 = 0; e2 < E / 2; ++e2) {
      if (e2 == E / 4) halfway();
      __builtin_amdgcn_sched_barrier(0);   // (conversions of several pairs at once take registers that there are not)
      unsigned x[8];
      pairs(e2, x);
      u32x4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        even[i] = pair_low(x[2 * i], x[2 * i + 1]);
        odd[i] = pair_high(x[2 * i], x[2 * i + 1]);
      }
      st.o[2 * e2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), __builtin_bit_cast(bf16x8, w[0][0]), st.o[2 * e2], 0, 0, 0);
      st.o[2 * e2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, w[0][0]), st.o[2 * e2 + 1], 0, 0, 0);
    }
  }
  template <typename HalfFn>
  __device__ static __forceinline__ void accumulate(State& st, const u32x4 (&w)[RT][1], const Values& v, HalfFn&& halfway) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = scale_of(v.scale[j >> 2], j & 3);
    add(st, w, [&](int e2, unsigned (&x)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = D == 128 ? two_values(v.c[j], f[j], e2) : two_values(v.c[j >> 1], f[j], 2 * (j & 1) + e2);
    }, halfway);
  }

  // ---- a block of the tree's own keys, bf16 (rows past the tree's end repeat its last one and are masked)
  struct TreeKeys { bf16x8 k[2][KS]; };
  struct TreeValues { unsigned v[NX][D / 32]; };
  __device__ static __forceinline__ void load_tree(TreeKeys& k, TreeValues& v, const char* kr, const char* vr, int64_t row_bytes, int t0, int last, int lane) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const char* src = kr + min(t0 + operand_key(kt, lane & 15), last) * row_bytes;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k.k[kt][ks] = *reinterpret_cast<const bf16x8*>(src + 2 * piece_channel(ks, lane));
    }
#pragma unroll
    for (int j = 0; j < NX; ++j) {
      const char* row = vr + min(t0 + first_key(lane) + key_of(j), last) * row_bytes;
      if constexpr (PLAIN) {   // of each half of the channels the lane's KS
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const char* src = row + 2 * (D / 2 * i + KS * (lane & 15));
          if constexpr (D == 128) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(src);
            v.v[j][2 * i] = w[0]; v.v[j][2 * i + 1] = w[1];
          } else {
            v.v[j][i] = *reinterpret_cast<const unsigned*>(src);
          }
        }
        continue;
      }
      const char* src = row + 2 * E * (lane & 15);
      if constexpr (D == 128) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[j][i] = w[i];
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(src);
        v.v[j][0] = w[0]; v.v[j][1] = w[1];
      }
    }
  }
  __device__ static __forceinline__ void score_tree(float (&s)[RT][NX], const TreeKeys& k, const u32x4 (&q)[RT][PIECES]) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.k[kt][ks], __builtin_bit_cast(bf16x8, q[0][ks]), r, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][4 * kt + i] = r[i];
    }
  }
  __device__ static __forceinline__ void accumulate_tree(State& st, const u32x4 (&w)[RT][1], const TreeValues& v) {
    add(st, w, [&](int e2, unsigned (&x)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = v.v[j][e2];
    }, [] {});
  }
  // the weight of a key of the block for the lane's row
  __device__ static __forceinline__ float weight_of(const u32x4 (&w)[1], int key, int lane) {
    const int at = PLAIN ? key & 7 : (key & 3) + 4 * (key >> 4);
    float own = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) own = at == j ? bf16_at(w[0][j >> 1], j & 1) : own;
    return __shfl(own, 16 * (PLAIN ? key >> 3 : (key >> 2) & 3) + (lane & 15));
  }
  // add(q, k, x): the sums of channel channel(q) + k get x
  __device__ static __forceinline__ void add_to(State& st, int, int q, int k, float x) {
    if constexpr (PLAIN && D == 64) st.o[2 * (q >> 1) + (k & 1)][2 * (q & 1) + (k >> 1)] += x;
    else st.o[4 * (q >> 2) + k][q & 3] += x;
  }
};

// ---------------------------------------------------------------------------------------------------------------------------
// Lane (col, h) = (lane % 32, lane / 32), tiles of 32 rows.
//   S^T: v_mfma_scale_f32_32x32x64_f8f6f4: every other block of 32 channels of key col; per 64 channels two products (hi, lo).
//   O^T: v_mfma_f32_32x32x16_bf16: D/32 channels (those are half a run of V's codes: run col % 16, half col / 16) of keys 16 h .. + 15.
//        Lanes col and col + 16 share runs: each loads eight of the keys and gives the other its half of them
//        (v_permlane16_swap_b32), instead of both loading all 16.
//   Row sums: v_mfma_f32_4x4x4_16b_bf16 with ones adds a lane's own weights four at a time; the halves of a row meet at the end.
template <int D, int TILES, bool PLAIN = false>
struct Form32 {
  static constexpr int HEAD_DIM = D, TILE = 32, RT = TILES, ROWS = 32 * TILES, NX = 16, E = D / 32, KB = D / 64;
  static constexpr int QUADS = D / 8;

  __device__ static __forceinline__ int row(int lane) { return lane & 31; }
  __device__ static __forceinline__ int first_key(int lane) { return 16 * (lane >> 5); }
  __device__ static constexpr int key_of(int j) { return j; }
  // the key that row m of the products' operand is, so that the scores of a lane are those of 16 keys in a row
  __device__ static __forceinline__ int operand_key(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }
  __device__ static __forceinline__ float row_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }

  struct State {
    f32x16 o[RT][E];   // entry r of tile e <-> operand row 8 (r / 4) + 4 h + r % 4, the channels of whose lane are values_channel(..) + e
    float m[RT];
    f32x4 l[RT];       // all entries equal; the lane's own keys
  };
  __device__ static __forceinline__ void clear(State& st, float m) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      st.m[t] = m;
      st.l[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[t][e][r] = 0.f;
    }
  }
  __device__ static __forceinline__ void rescale(State& st, int t, float a) {
    st.l[t] *= a;
#pragma unroll
    for (int e = 0; e < E; ++e) st.o[t][e] *= a;
  }
  __device__ static __forceinline__ float row_sum(const State& st, int t) { return st.l[t][0] + __shfl_xor(st.l[t][0], 32); }
  // D = 128: quad q is entry q of the four tiles. D = 64: entries q and q + 8 of the two (q < 8), or 2 q and 2 q + 1, whose channels follow one another.
  __device__ static __forceinline__ f32x4 quad(const State& st, int t, int q) {
    if constexpr (D == 128) return f32x4{st.o[t][0][q], st.o[t][1][q], st.o[t][E - 2][q], st.o[t][E - 1][q]};
    else if constexpr (PLAIN) return f32x4{st.o[t][0][2 * q], st.o[t][1][2 * q], st.o[t][0][2 * q + 1], st.o[t][1][2 * q + 1]};
    else return f32x4{st.o[t][0][q], st.o[t][1][q], st.o[t][0][q + 8], st.o[t][1][q + 8]};
  }
  // first channel of a lane of V: 2 E channels a run, E of them the lane's
  __device__ static constexpr int values_channel(int col) { return PLAIN ? E * col : 2 * E * (col & 15) + E * (col >> 4); }
  __device__ static __forceinline__ int channel(int q, int lane) {
    const int r = PLAIN && D == 64 ? 2 * q : q;
    return values_channel(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3));
  }
  __device__ static __forceinline__ void add_to(State& st, int t, int q, int k, float x) {
    if constexpr (D == 128) st.o[t][k][q] += x;
    else if constexpr (PLAIN) st.o[t][k & 1][2 * q + (k >> 1)] += x;
    else st.o[t][k & 1][q + 8 * (k >> 1)] += x;
  }

  static constexpr int PIECES = D / 16;
  __device__ static __forceinline__ int piece_channel(int i, int lane) { return 64 * (i >> 2) + 32 * ((i >> 1) & 1) + 16 * (lane >> 5) + 8 * (i & 1); }
  struct Query {
    i32x8 hi[RT][KB], lo[RT][KB];
    int scale[RT];   // hi's in the first byte, lo's in the second
  };
  __device__ static __forceinline__ void split(Query& q, int t, const u32x4 (&piece)[PIECES], int) {
    unsigned x[4 * PIECES];
#pragma unroll
    for (int i = 0; i < 4 * PIECES; ++i) x[i] = piece[i >> 2][i & 3];
    unsigned top = top_of(x);
    top = max(top, (unsigned)__shfl_xor((int)top, 32));
    int hi[2 * PIECES], lo[2 * PIECES], s_hi, s_lo;
    split_row(x, top, hi, lo, s_hi, s_lo);
#pragma unroll
    for (int i = 0; i < 8 * KB; ++i) { q.hi[t][i >> 3][i & 7] = hi[i]; q.lo[t][i >> 3][i & 7] = lo[i]; }
    q.scale[t] = s_hi | s_lo << 8;
  }

  struct Keys {
    u32x4 c[KB];
    unsigned scale[KB];
  };
  struct Values {
    unsigned c[4 * KB], scale[4];   // eight of the lane's 16 keys, the scales of all
  };
  static constexpr bool HEADS_FIRST = false;   // the order of a call's units
  // where a block's codes and scales start in a head's part of a page, in which a lane's Offsets are counted
  __device__ static constexpr int head_bytes(int P) { return page_head_bytes(D, P); }
  __device__ static __forceinline__ unsigned block_codes(unsigned in_page) { return in_page * (D / 2); }
  __device__ static __forceinline__ unsigned block_scales(unsigned in_page) { return in_page; }
  struct Offsets { unsigned k, ks, v, vs; };
  template <bool WIDE>
  __device__ static __forceinline__ Offsets offsets(int lane, int P) {
    const int col = lane & 31, h = lane >> 5, late = col >> 4, codes = page_code_bytes(D, P), scales = page_scale_bytes(D, P);
    const int key = operand_key(col) & (WIDE ? 31 : 15);
    Offsets o;
    o.k = (unsigned)(key * (D / 2) + h * 16);
    o.ks = (unsigned)(2 * codes + h * P + key);
    o.v = (unsigned)(codes + (WIDE ? h * 16 * (D / 2) : 0) + late * 8 * (D / 2) + (col & 15) * 16);   // (pieces of eight keys: 256 bytes, or two times)
    o.vs = (unsigned)(2 * codes + scales + (2 * E * (col & 15) / 32) * P + (WIDE ? 16 * h : 0));
    return o;
  }
  template <bool WIDE>
  __device__ static __forceinline__ void load_keys(Keys& x, const BlockPlace<WIDE>& at, const Offsets& off, int lane, int P) {
    const unsigned k = here(off.k), ks = here(off.ks);
    const int half = !WIDE && (here(lane) & 4) ? 1 : 0;   // (of a narrow block: operand_key)
    GlobalBytes const code = half ? at.code[BlockPlace<WIDE>::HALVES - 1] : at.code[0], scale = half ? at.scale[BlockPlace<WIDE>::HALVES - 1] : at.scale[0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      x.c[kb] = fetch<u32x4>(code + k + 32 * kb);
      x.scale[kb] = fetch<uint8_t>(scale + 2 * kb * P + ks);
    }
  }
  template <bool WIDE>
  __device__ static __forceinline__ void load_values(Values& x, const BlockPlace<WIDE>& at, const Offsets& off, int lane) {
    const unsigned v = here(off.v), vs = here(off.vs);
    const int half = !WIDE && (here(lane) & 32) ? 1 : 0;
    GlobalBytes const code = half ? at.code[BlockPlace<WIDE>::HALVES - 1] : at.code[0], scale = half ? at.scale[BlockPlace<WIDE>::HALVES - 1] : at.scale[0];
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      const u32x4 w = fetch<u32x4>(code + v + 256 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x.c[4 * i + k] = w[k];
    }
    const u32x4 w = fetch<u32x4>(scale + vs);
#pragma unroll
    for (int k = 0; k < 4; ++k) x.scale[k] = w[k];
  }
  __device__ static __forceinline__ void mask_values(Values& x, unsigned vis, int lane) {
    const unsigned own = vis >> here(first_key(lane));
#pragma unroll
    for (int j = 0; j < NX; ++j)
      if (!((own >> key_of(j)) & 1u)) x.scale[j >> 2] = (x.scale[j >> 2] & ~(0xffu << (8 * (j & 3)))) | (0x7fu << (8 * (j & 3)));
  }
  __device__ static __forceinline__ void score(float (&s)[RT][NX], const Keys& keys, const Query& q) {
    f32x16 r[RT];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const u32x4 c = keys.c[kb];
      const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x16 before;
#pragma unroll
        for (int i = 0; i < 16; ++i) before[i] = kb == 0 ? 0.f : r[t][i];
        r[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.hi[t][kb], before, 4 /* a: fp4 */, 0 /* b: e4m3 */, 0, (int)keys.scale[kb], 0, q.scale[t]);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)
        r[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.lo[t][kb], r[t], 4, 0, 0, (int)keys.scale[kb], 1 /* the second byte */, q.scale[t]);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int j = 0; j < NX; ++j) s[t][j] = r[t][j];
  }
  // rows(s, i, x0, x1): channel pairs of keys 2 i and 2 i + 1 of the lane's eight keys s
  template <typename PairFn, typename HalfFn>
  __device__ static __forceinline__ void add(State& st, const u32x4 (&w)[RT][2], PairFn&& rows, HalfFn&& halfway) {
    u32x2 one_bits = {0x3f803f80u, 0x3f803f80u};
    asm volatile("" : "+v"(one_bits));   // (kept, not made again from scalars for every product)
    const s16x4 ones = __builtin_bit_cast(s16x4, one_bits);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s == 1) halfway();
      __builtin_amdgcn_sched_barrier(0);
      u32x4 a[E];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        unsigned x0[E / 2], x1[E / 2];
        rows(s, i, x0, x1);
#pragma unroll
        for (int e2 = 0; e2 < E / 2; ++e2) {
          a[2 * e2][i] = pair_low(x0[e2], x1[e2]);
          a[2 * e2 + 1][i] = pair_high(x0[e2], x1[e2]);
        }
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int e = 0; e < E; ++e) st.o[t][e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[e]), __builtin_bit_cast(bf16x8, w[t][s]), st.o[t][e], 0, 0, 0);
        const u32x2 front = {w[t][s][0], w[t][s][1]}, back = {w[t][s][2], w[t][s][3]};
        st.l[t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, front), st.l[t], 0, 0, 0);
        st.l[t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, back), st.l[t], 0, 0, 0);
      }
    }
  }
  template <typename HalfFn>
  __device__ static __forceinline__ void accumulate(State& st, const u32x4 (&w)[RT][2], const Values& v, HalfFn&& halfway) {
    // each piece's half for the lower lanes of a pair and for the upper ones, then the exchange: after it `mine[s]` are the lane's channels of keys 8 s .. 8 s + 7 of its 16
    unsigned mine[2][2 * KB];
#pragma unroll
    for (int i = 0; i < 2 * KB; ++i) {
      unsigned low, high;
      if constexpr (D == 128) {
        low = pair_low(v.c[2 * i], v.c[2 * i + 1]);
        high = pair_high(v.c[2 * i], v.c[2 * i + 1]);
      } else {
        low = __builtin_amdgcn_perm(v.c[2 * i + 1], v.c[2 * i], 0x06040200u);
        high = __builtin_amdgcn_perm(v.c[2 * i + 1], v.c[2 * i], 0x07050301u);
      }
      const auto both = __builtin_amdgcn_permlane16_swap(low, high, false, false);
      mine[0][i] = both[0];
      mine[1][i] = both[1];
    }
    add(st, w, [&](int s, int i, unsigned (&x0)[E / 2], unsigned (&x1)[E / 2]) {
      const unsigned scales = v.scale[2 * s + (i >> 1)];
      const float f0 = scale_of(scales, 2 * (i & 1)), f1 = scale_of(scales, 2 * (i & 1) + 1);
#pragma unroll
      for (int e2 = 0; e2 < E / 2; ++e2) {
        if constexpr (D == 128) {   // a word: two keys of two bytes
          x0[e2] = two_values(mine[s][i], f0, e2);
          x1[e2] = two_values(mine[s][i], f1, 2 + e2);
        } else {                    // a word: four keys of one byte
          x0[e2] = two_values(mine[s][i >> 1], f0, 2 * (i & 1));
          x1[e2] = two_values(mine[s][i >> 1], f1, 2 * (i & 1) + 1);
        }
      }
    }, halfway);
  }

  struct TreeKeys { bf16x8 k[PIECES]; };
  struct TreeValues { unsigned v[NX][E / 2]; };
  __device__ static __forceinline__ void load_tree(TreeKeys& k, TreeValues& v, const char* kr, const char* vr, int64_t row_bytes, int t0, int last, int lane) {
    const char* src = kr + min(t0 + operand_key(lane & 31), last) * row_bytes;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) k.k[i] = *reinterpret_cast<const bf16x8*>(src + 2 * piece_channel(i, lane));
#pragma unroll
    for (int j = 0; j < NX; ++j) {
      const char* from = vr + min(t0 + first_key(lane) + key_of(j), last) * row_bytes + 2 * values_channel(lane & 31);
      if constexpr (D == 128) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(from);
        v.v[j][0] = w[0]; v.v[j][E / 2 - 1] = w[1];
      } else {
        v.v[j][0] = *reinterpret_cast<const unsigned*>(from);
      }
    }
  }
  __device__ static __forceinline__ void score_tree(float (&s)[RT][NX], const TreeKeys& k, const u32x4 (&q)[RT][PIECES]) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x16 r;
#pragma unroll
      for (int j = 0; j < 16; ++j) r[j] = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.k[i], __builtin_bit_cast(bf16x8, q[t][i]), r, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < NX; ++j) s[t][j] = r[j];
    }
  }
  __device__ static __forceinline__ void accumulate_tree(State& st, const u32x4 (&w)[RT][2], const TreeValues& v) {
    add(st, w, [&](int s, int i, unsigned (&x0)[E / 2], unsigned (&x1)[E / 2]) {
#pragma unroll
      for (int e2 = 0; e2 < E / 2; ++e2) {
        x0[e2] = v.v[8 * s + 2 * i][e2];
        x1[e2] = v.v[8 * s + 2 * i + 1][e2];
      }
    }, [] {});
  }
  __device__ static __forceinline__ float weight_of(const u32x4 (&w)[2], int key, int lane) {
    float own = 0.f;
#pragma unroll
    for (int j = 0; j < NX; ++j) own = (key & 15) == j ? bf16_at(w[j >> 3][(j & 7) >> 1], j & 1) : own;
    return __shfl(own, 32 * (key >> 4) + (lane & 31));
  }
};

}  // namespace fspad_detail

#endif
