// The two forms of paged_forms.h over a paged 8-bit cache: what lanes hold of a 32-key block of e4m3 codes, and the products with it.
// Internal to the library. gfx950 (CDNA4) only.
//
// Scores take K's codes and scale as they are, on the block-scaled products, against the same two fp8 rows that hold a query. V's codes lie key
// after key in their pages, channel by channel: a lane loads an operand of the products as it is, and v_cvt_scalef32_pk_bf16_fp8 makes bf16 of two
// codes and the block's scale, exactly. Nothing is turned.
#ifndef FSPAD_PAGED_FORMS_FP8_H
#define FSPAD_PAGED_FORMS_FP8_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_forms.h"
#include "paged_layout.h"

namespace fspad_detail {

// Eight codes (two words) to bf16, times the block's scale.
__device__ __forceinline__ bf16x8 eight_values(unsigned low, unsigned high, float scale) {
  u32x4 x;
  x[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false));
  x[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true));
  x[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false));
  x[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true));
  return __builtin_bit_cast(bf16x8, x);
}

// Bytes of all ones where the lowest four bits are.
__device__ __forceinline__ unsigned bytes_of(unsigned bits) { return (((bits & 15u) * 0x00204081u) & 0x01010101u) * 0xffu; }

// What both forms share: one scale byte of K and one of V a block.
template <int D>
struct Fp8Block {
  static constexpr bool HEADS_FIRST = true;
  __device__ static constexpr int head_bytes(int P) { return page_head_bytes_fp8(D, P); }
  __device__ static __forceinline__ unsigned block_codes(unsigned in_page) { return in_page * D; }
  __device__ static __forceinline__ unsigned block_scales(unsigned in_page) { return in_page / kFp8BlockTokens; }
  struct Offsets { unsigned k, v, ks; };
};

// Lane (col, g4) = (lane % 16, lane / 16).
//   S^T: v_mfma_scale_f32_16x16x128_f8f6f4: channels 16 g4 .. and, D = 128, 64 + 16 g4 .. of a key; D = 64: K's 64 channels twice in its 128.
//   O^T: v_mfma_f32_16x16x32_bf16: D/16 channels of keys 8 g4 .. 8 g4 + 7.
template <int D>
struct Form16Fp8 : Form16<D, true>, Fp8Block<D> {
  using Base = Form16<D, true>;
  using Block = Fp8Block<D>;
  using Block::HEADS_FIRST;
  using Block::head_bytes;
  using Block::block_codes;
  using Block::block_scales;
  using typename Block::Offsets;
  using typename Base::Query;
  using typename Base::State;
  static constexpr int RT = 1, NX = 8, E = Base::E, KS = Base::KS, HALVES = D / 64;

  struct Keys {
    u32x4 c[2][HALVES];
    unsigned scale;
  };
  struct Values {
    u32x2 c[E];
    unsigned scale;
  };
  template <bool WIDE>
  __device__ static __forceinline__ Offsets offsets(int lane, int P) {
    const int col = lane & 15, g4 = lane >> 4;
    Offsets o;
    o.k = (unsigned)((g4 * 32 + Base::operand_key(0, col)) * 16);
    o.v = (unsigned)(P * D + ((g4 >> 1) * 32 + col) * 16 + (g4 & 1) * 8);
    o.ks = (unsigned)(2 * P * D);
    return o;
  }
  __device__ static __forceinline__ void load_keys(Keys& x, const BlockPlace<true>& at, const Offsets& off, int, int) {
    const unsigned k = here(off.k), ks = here(off.ks);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)   // (four keys further on)
#pragma unroll
      for (int i = 0; i < HALVES; ++i) x.c[kt][i] = fetch<u32x4>(at.code[0] + k + 64 * kt + 2048 * i);
    x.scale = fetch<uint8_t>(at.scale[0] + ks);
  }
  __device__ static __forceinline__ void load_values(Values& x, const BlockPlace<true>& at, const Offsets& off, int) {
    const unsigned v = here(off.v), ks = here(off.ks);
#pragma unroll
    for (int e = 0; e < E; ++e) x.c[e] = fetch<u32x2>(at.code[0] + v + 1024 * (e % KS) + 256 * (e / KS));
    x.scale = fetch<uint8_t>(at.scale[0] + ks + kFp8VScales);
  }
  // Keys that are not there: codes of zero, under any scale if none is.
  __device__ static __forceinline__ void mask_values(Values& x, unsigned vis, int lane) {
    const unsigned own = vis >> here(Base::first_key(lane)), low = bytes_of(own), high = bytes_of(own >> 4);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x.c[e][0] &= low;
      x.c[e][1] &= high;
    }
    if (vis == 0) x.scale = 127;
  }
  __device__ static __forceinline__ void score(float (&s)[RT][NX], const Keys& keys, const Query& q) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const u32x4 c = keys.c[kt][0], d = keys.c[kt][HALVES - 1];
      const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], (int)d[0], (int)d[1], (int)d[2], (int)d[3]};
      f32x4 r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.v[0][0], f32x4{0.f, 0.f, 0.f, 0.f}, 0 /* a: e4m3 */, 0 /* b: e4m3 */, 0, (int)keys.scale, 0,
                                                                 q.scale[0]);
      if constexpr (D == 128)
        r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.v[0][D / 64 - 1], r, 0, 0, 0, (int)keys.scale, 1 /* the second byte */, q.scale[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][4 * kt + i] = r[i];
    }
  }
  template <typename HalfFn>
  __device__ static __forceinline__ void accumulate(State& st, const u32x4 (&w)[RT][1], const Values& v, HalfFn&& halfway) {
    const float scale = scale_of(v.scale, 0);
    Base::add_weights(st, w);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e == E / 2) halfway();
      st.o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_values(v.c[e][0], v.c[e][1], scale), __builtin_bit_cast(bf16x8, w[0][0]), st.o[e], 0, 0, 0);
    }
  }
};

// Lane (col, h) = (lane % 32, lane / 32), tiles of 32 rows.
//   S^T: v_mfma_scale_f32_32x32x64_f8f6f4: channels 64 i + 16 h .. and 64 i + 32 + 16 h .. of a key; per 64 channels two products (hi, lo).
//   O^T: v_mfma_f32_32x32x16_bf16: D/32 channels of keys 16 h .. + 15.
template <int D, int TILES>
struct Form32Fp8 : Form32<D, TILES, true>, Fp8Block<D> {
  using Base = Form32<D, TILES, true>;
  using Block = Fp8Block<D>;
  using Block::HEADS_FIRST;
  using Block::head_bytes;
  using Block::block_codes;
  using Block::block_scales;
  using typename Block::Offsets;
  using typename Base::Query;
  using typename Base::State;
  static constexpr int RT = TILES, NX = 16, E = Base::E, KB = Base::KB;

  struct Keys {
    u32x4 c[KB][2];
    unsigned scale;
  };
  struct Values {
    u32x4 c[E];
    unsigned scale;
  };
  template <bool WIDE>
  __device__ static __forceinline__ Offsets offsets(int lane, int P) {
    const int col = lane & 31, h = lane >> 5;
    Offsets o;
    o.k = (unsigned)((h * 32 + Base::operand_key(col)) * 16);
    o.v = (unsigned)(P * D + lane * 16);
    o.ks = (unsigned)(2 * P * D);
    return o;
  }
  __device__ static __forceinline__ void load_keys(Keys& x, const BlockPlace<true>& at, const Offsets& off, int, int) {
    const unsigned k = here(off.k), ks = here(off.ks);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 2; ++i) x.c[kb][i] = fetch<u32x4>(at.code[0] + k + 2048 * kb + 1024 * i);
    x.scale = fetch<uint8_t>(at.scale[0] + ks);
  }
  __device__ static __forceinline__ void load_values(Values& x, const BlockPlace<true>& at, const Offsets& off, int) {
    const unsigned v = here(off.v), ks = here(off.ks);
#pragma unroll
    for (int e = 0; e < E; ++e) x.c[e] = fetch<u32x4>(at.code[0] + v + 1024 * e);
    x.scale = fetch<uint8_t>(at.scale[0] + ks + kFp8VScales);
  }
  __device__ static __forceinline__ void mask_values(Values& x, unsigned vis, int lane) {
    const unsigned own = vis >> here(Base::first_key(lane));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned there = bytes_of(own >> (4 * i));
#pragma unroll
      for (int e = 0; e < E; ++e) x.c[e][i] &= there;
    }
    if (vis == 0) x.scale = 127;
  }
  __device__ static __forceinline__ void score(float (&s)[RT][NX], const Keys& keys, const Query& q) {
    f32x16 r[RT];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const u32x4 c = keys.c[kb][0], d = keys.c[kb][1];
      const i32x8 a = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], (int)d[0], (int)d[1], (int)d[2], (int)d[3]};
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x16 before;
#pragma unroll
        for (int i = 0; i < 16; ++i) before[i] = kb == 0 ? 0.f : r[t][i];
        r[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.hi[t][kb], before, 0 /* a: e4m3 */, 0 /* b: e4m3 */, 0, (int)keys.scale, 0, q.scale[t]);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)
        r[t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.lo[t][kb], r[t], 0, 0, 0, (int)keys.scale, 1 /* the second byte */, q.scale[t]);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int j = 0; j < NX; ++j) s[t][j] = r[t][j];
  }
  template <typename HalfFn>
  __device__ static __forceinline__ void accumulate(State& st, const u32x4 (&w)[RT][2], const Values& v, HalfFn&& halfway) {
    const float scale = scale_of(v.scale, 0);
    u32x2 one_bits = {0x3f803f80u, 0x3f803f80u};
    asm volatile("" : "+v"(one_bits));   // (kept, not made again from scalars for every product)
    const s16x4 ones = __builtin_bit_cast(s16x4, one_bits);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s == 1) halfway();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bf16x8 a = eight_values(v.c[e][2 * s], v.c[e][2 * s + 1], scale);
#pragma unroll
        for (int t = 0; t < RT; ++t) st.o[t][e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, w[t][s]), st.o[t][e], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const u32x2 front = {w[t][s][0], w[t][s][1]}, back = {w[t][s][2], w[t][s][3]};
        st.l[t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, front), st.l[t], 0, 0, 0);
        st.l[t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, back), st.l[t], 0, 0, 0);
      }
    }
  }
};

}  // namespace fspad_detail

#endif
