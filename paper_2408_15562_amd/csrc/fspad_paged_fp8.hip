// Store and load of the paged 8-bit cache (include/fspad.h, "Paged 8-bit cache"). The attention over it is in fspad_attn_paged_fp8.hip. gfx950 (CDNA4) only.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256, kBlock = kFp8BlockTokens, kGroup = 16;   // tokens of a block, of a run of V's codes

struct RowsParams {
  char* k;               // [rows] x [Hkv] x D bf16: read by the store, written by the load
  char* v;
  const int32_t* slots;
  int32_t* row_of;       // store of many rows: per slot of the pool, the row that goes there (what no row has written is anything)
  char* pages;
  int64_t row_stride, head_stride;   // bytes
  int64_t page_stride;
  int32_t rows, n_slots, page_shift;
};

// Where channel c of token t of a block lies among the block's codes of K.
__device__ __forceinline__ int k_code_at(int t, int c) { return ((c >> 4) * kBlock + t) * 16 + (c & 15); }
template <int D>
__device__ __forceinline__ char* head_of(const RowsParams& p, int slot, int head) {
  return p.pages + (int64_t)(slot >> p.page_shift) * p.page_stride + (int64_t)head * page_head_bytes_fp8(D, 1 << p.page_shift);
}

// A block's scale byte from the bits of its largest finite magnitude (bf16 without the sign): the smallest s with a <= 448 * 2^(s-127), 448
// being 1.75 * 2^8. 10 .. 246 keep every value a normal, finite bf16: the smallest element is 2^-9, the largest becomes 7 * 2^125.
constexpr unsigned kTopBits = 0x7f60;   // that one's
__device__ __forceinline__ int scale_for(unsigned top) {
  const int s = (int)(top >> 7) - 8 + ((top & 0x7f) > 0x60 ? 1 : 0);
  return min(max(s, 10), 246);
}
__device__ __forceinline__ float as_scale(int s) { return __builtin_bit_cast(float, s << 23); }

__device__ __forceinline__ unsigned finite_or_zero(unsigned magnitude) { return magnitude < 0x7f80u ? magnitude : 0u; }
__device__ __forceinline__ unsigned at_most_top(unsigned bits) { return (bits & 0x7fffu) < 0x7f80u ? (bits & 0x8000u) | min(bits & 0x7fffu, kTopBits) : bits; }

// Four channels to codes: rounded to nearest, ties to even. WILD: some are NaN or infinite, which become NaN (all bits below the sign).
template <bool WILD>
__device__ __forceinline__ unsigned encode4(unsigned low, unsigned high, float scale) {
  s16x2 c = {0, 0};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, low), scale, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, high), scale, true);
  unsigned codes = __builtin_bit_cast(unsigned, c);
  if constexpr (WILD) {
    codes |= (low & 0x7f80u) == 0x7f80u ? 0x7fu : 0u;
    codes |= (low & 0x7f800000u) == 0x7f800000u ? 0x7f00u : 0u;
    codes |= (high & 0x7f80u) == 0x7f80u ? 0x7f0000u : 0u;
    codes |= (high & 0x7f800000u) == 0x7f800000u ? 0x7f000000u : 0u;
  }
  return codes;
}
__device__ __forceinline__ u32x2 decode4(unsigned codes, float scale) {
  return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
// Codes under one scale, rounded again under a larger one.
__device__ __forceinline__ unsigned again4(unsigned codes, float had, float scale) {
  const u32x2 x = decode4(codes, had);
  return encode4<true>(x[0], x[1], scale);
}

// ---------------------------------------------------------------------------------------------
// Store. A block's scale is that of all its tokens, so whoever stores to a block (of a head) has all of a call's rows of it: looks for
// them, forms the largest magnitude, rounds, and where the scale of a block that holds tokens grows rounds those again. The rows of a block
// may stand anywhere in the call. A workgroup looks after some neighbouring rows, block by block. Are all of a block's tokens in neighbouring rows (a prompt's are), it sees that
// from the slots of these and some rows around them. Else it goes through all of the call's slots, or, of many rows, through
// a list by slot that a launch before this one writes. The block is that workgroup's whose rows have the block's lowest token.
//
// What bounds it: memory, for many rows. 8191 rows of 32 heads, D = 128 (201 MB), 37 us where all of it stays in the memory-side cache, 55 behind a load of as many rows,
// whose 134 MB are written back meanwhile (36 us without reads, 41 without writes; one, two or four heads at once, more heads a workgroup, the next head's rows asked for ahead:
// 54 to 57). A few rows: launch and trips, 4.7 us.
//
// Groups of 256 threads have a head each. Every thread has a piece of K and of V the channels of four neighbouring tokens that make four neighbouring bytes of
// D/32 places: what it rounds it stores, whole lines a wavefront.
// At most, without the list. Rows of trees of 60 nodes, 5 of them stored, 8 heads, both ways: 3840 rows 9.8 us without and 8.0 with it, 15360 35.6 and 14.7; a prompt of 8191 rows of 32 heads 90
// either way.
constexpr int kScanRows = 2048;
constexpr int kMostChunk = 32;     // rows that a workgroup looks after
constexpr int kWindow = kMostChunk + 2 * (kBlock - 1);   // and sees
// Rows are taken together down to so many workgroups. 1024, 2048, 4096: accepted paths of 4 trees, 52 heads (with their load) 8.5, 8.9, 9.7 us; a token of 512 sequences, 8 heads, 14.7, 13.5, 11.6
constexpr int kChunkWorkgroups = 2048;
constexpr int kEnoughWorkgroups = 1024, kHeadsAtOnce = 2, kMostHeads = 4;

__global__ __launch_bounds__(kThreads) void kv_rows_of_slots_kernel(const RowsParams p) {
  const int row = blockIdx.x * kThreads + threadIdx.x;
  if (row >= p.rows) return;
  const int slot = p.slots[row];
  if ((unsigned)slot < (unsigned)p.n_slots) p.row_of[slot] = row;
}

template <int HEADS>
struct StoreShared {
  int slot[kWindow];        // of rows row0 - 31 .., -1 outside the call or the pool
  int member[kBlock];       // the row of each token of the block at hand
  unsigned top[2][HEADS][2][kThreads / 64];
};

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// Largest magnitude (bits) of some words of two values each. Magnitudes of bf16 compare as integers, infinity and NaN (from 0x7f80 on) above the rest.
template <int N>
__device__ __forceinline__ unsigned top_of(const unsigned (&w)[N]) {
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  return max((unsigned)m[0], (unsigned)m[1]);
}
template <int N>
__device__ __forceinline__ unsigned finite_top_of(const unsigned (&w)[N]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) top = max(top, max(finite_or_zero(w[i] & 0x7fffu), finite_or_zero((w[i] >> 16) & 0x7fffu)));
  return top;
}

__device__ __forceinline__ unsigned bytes_of(unsigned bits) { return (((bits & 15u) * 0x00204081u) & 0x01010101u) * 0xffu; }

// A thread's part of a block of one head: of K, 8 channels of two tokens, which it makes 16 of one with its neighbour (loads of 16 channels a lane, in two
// halves, would ask for every line twice); of V, the E channels of four tokens.
// ALL: every token of the block has a row.
template <int D, bool ALL>
struct StorePart {
  static constexpr int LANES = D / 8, E = D / 32, VW = E / 2;   // lanes of a token of K, words of one of V
  static constexpr bool SOME = kBlock * LANES < 2 * kThreads;   // (K has no part for some threads)

  // what is the same for all heads
  struct Place {
    const char *k[2], *v[4];
    int k_at, v_at;                 // bytes from the block's codes on
    unsigned has_k, own_k, has_v;   // bit i: token i of two (of four) is there; whether the one is that the thread stores
  };
  __device__ static __forceinline__ Place place(const RowsParams& p, const int* member, unsigned there) {
    const int tid = threadIdx.x % kThreads, pair = tid / LANES, lane = tid % LANES;
    const int first = 16 * ((tid >> 6) & 1) + 4 * (tid & 3), row = 16 * (tid >> 7) + ((tid >> 2) & 15);
    const bool has_part = !SOME || 2 * pair < kBlock;
    Place x;
    x.has_k = !has_part ? 0u : ALL ? 3u : (there >> (2 * pair)) & 3u;
    x.own_k = (x.has_k >> (lane & 1)) & 1u;
    x.has_v = ALL ? 15u : (there >> first) & 15u;
#pragma unroll
    for (int i = 0; i < 2; ++i) x.k[i] = p.k + ((x.has_k >> i) & 1u ? member[2 * pair + i] : 0) * p.row_stride + lane * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = p.v + ((x.has_v >> i) & 1u ? member[first + i] : 0) * p.row_stride + row * (2 * E);
    x.k_at = has_part ? ((lane >> 1) * kBlock + 2 * pair + (lane & 1)) * 16 : -1;
    x.v_at = ((first >> 4) * 32 + row) * 16 + (first & 15);
    return x;
  }

  unsigned k[8], v[4 * VW];   // (k: four words a token)
  int had[2];

  // head: bytes from a row's first head on
  __device__ __forceinline__ void load(const Place& x, int64_t head, bool begun, const unsigned char* scales) {
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = 0;
#pragma unroll
    for (int i = 0; i < 4 * VW; ++i) v[i] = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if ((ALL && !SOME) || ((x.has_k >> i) & 1u)) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(x.k[i] + head);
#pragma unroll
        for (int j = 0; j < 4; ++j) k[4 * i + j] = w[j];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (ALL || ((x.has_v >> i) & 1u)) {
        if constexpr (E == 4) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(x.v[i] + head);
          v[VW * i] = w[0];
          v[VW * i + VW - 1] = w[1];
        } else {
          v[i] = *reinterpret_cast<const unsigned*>(x.v[i] + head);
        }
      }
    had[0] = had[1] = 0;
    if (!ALL && !begun) {
      had[0] = scales[0];
      had[1] = scales[kFp8VScales];
    }
  }

  template <bool WILD>
  __device__ __forceinline__ void encode(u32x4& kc, unsigned (&vc)[E], float k_scale, float v_scale) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) kc[i] = encode4<WILD>(k[2 * i], k[2 * i + 1], k_scale);   // the first token's two words, the second one's
    // lanes of even numbers keep the first token and get the other half of its channels, the others the second one
    const bool odd = threadIdx.x & 1;
    const unsigned give0 = odd ? kc[0] : kc[2], give1 = odd ? kc[1] : kc[3];
    const unsigned get0 = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give0, 0xB1, 0xf, 0xf, true);   // quad_perm 1,0,3,2
    const unsigned get1 = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give1, 0xB1, 0xf, 0xf, true);
    kc = odd ? u32x4{get0, get1, kc[2], kc[3]} : u32x4{kc[0], kc[1], get0, get1};
    // V: from channel after channel of a token to token after token of a channel
    if constexpr (E == 4) {
      unsigned a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = encode4<WILD>(v[VW * i], v[VW * i + VW - 1], v_scale);
      const unsigned low01 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), high01 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
      const unsigned low23 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), high23 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
      vc[0] = __builtin_amdgcn_perm(low23, low01, 0x05040100u);
      vc[1] = __builtin_amdgcn_perm(low23, low01, 0x07060302u);
      vc[E - 2] = __builtin_amdgcn_perm(high23, high01, 0x05040100u);
      vc[E - 1] = __builtin_amdgcn_perm(high23, high01, 0x07060302u);
    } else {
      const unsigned w01 = encode4<WILD>(v[0], v[1], v_scale), w23 = encode4<WILD>(v[2], v[3], v_scale);
      vc[0] = __builtin_amdgcn_perm(w23, w01, 0x06040200u);
      vc[E - 1] = __builtin_amdgcn_perm(w23, w01, 0x07050301u);
    }
  }

  // top: of the whole block, the finite ones'; wild: the thread has others
  __device__ __forceinline__ void store(const Place& x, const unsigned (&top)[2], bool wild, bool begun, char* k_codes, char* v_codes, unsigned char* scales) {
    const int tid = threadIdx.x % kThreads;
    int s[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) s[kv] = max(scale_for(top[kv]), had[kv]);
    if (__builtin_expect(max(top[0], top[1]) > kTopBits, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = at_most_top(k[i] & 0xffffu) | at_most_top(k[i] >> 16) << 16;
#pragma unroll
      for (int i = 0; i < 4 * VW; ++i) v[i] = at_most_top(v[i] & 0xffffu) | at_most_top(v[i] >> 16) << 16;
    }
    u32x4 kc;
    unsigned vc[E];
    if (__builtin_expect(__any(wild), 0)) encode<true>(kc, vc, as_scale(s[0]), as_scale(s[1]));
    else encode<false>(kc, vc, as_scale(s[0]), as_scale(s[1]));
    u32x4* const k_to = reinterpret_cast<u32x4*>(k_codes + x.k_at);
    unsigned* const v_to = reinterpret_cast<unsigned*>(v_codes + x.v_at);
    if constexpr (ALL) {
      if (!SOME || x.own_k) *k_to = kc;
#pragma unroll
      for (int e = 0; e < E; ++e) v_to[256 * e] = vc[e];
      if (tid < 2) scales[kFp8VScales * tid] = (unsigned char)(tid == 0 ? s[0] : s[1]);
    } else {
      const bool k_grown = !begun && s[0] > had[0], v_grown = !begun && s[1] > had[1];
      if (x.own_k) {
        *k_to = kc;
      } else if (k_grown && x.k_at >= 0) {
        u32x4 c = *k_to;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = again4(c[i], as_scale(had[0]), as_scale(s[0]));
        *k_to = c;
      }
      if (x.has_v || v_grown) {
        if (x.has_v != 15u) {   // beside bytes of other tokens
          const unsigned bytes = bytes_of(x.has_v);
          unsigned was[E];
#pragma unroll
          for (int e = 0; e < E; ++e) was[e] = v_to[256 * e];
#pragma unroll
          for (int e = 0; e < E; ++e) vc[e] = (vc[e] & bytes) | ((v_grown ? again4(was[e], as_scale(had[1]), as_scale(s[1])) : was[e]) & ~bytes);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) v_to[256 * e] = vc[e];
      }
      if (tid < 2 && (begun || (tid == 0 ? k_grown : v_grown))) scales[kFp8VScales * tid] = (unsigned char)(tid == 0 ? s[0] : s[1]);
    }
  }
};

// One block of heads head0, .. < head1, HEADS of them at once. there: which of its tokens have a row (sh.member).
template <int D, bool ALL, int HEADS>
__device__ __forceinline__ void store_heads(const RowsParams& p, StoreShared<HEADS>& sh, unsigned there, int slot0, int head0, int head1) {
  using Part = StorePart<D, ALL>;
  const int P = 1 << p.page_shift, nth = (slot0 & (P - 1)) / kBlock, tid = threadIdx.x % kThreads, own = HEADS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  const bool begun = there & 1u;
  const typename Part::Place place = Part::place(p, sh.member, there);
#pragma unroll 1
  for (int first = head0, round = 0; first < head1; first += HEADS, round ^= 1) {
    const int head = min(first + own, head1 - 1);   // (a group that has none left does the last one's again, and does not store it)
    char* const at = head_of<D>(p, slot0, head);
    char* const codes = at + nth * (kBlock * D);
    unsigned char* const scales = (unsigned char*)at + 2 * P * D + nth;
    Part part;
    part.load(place, head * p.head_stride, begun, scales);
    unsigned top[2] = {top_of(part.k), top_of(part.v)};
    const bool wild = max(top[0], top[1]) >= 0x7f80u;
    if (__builtin_expect(__any(wild), 0)) {
      top[0] = finite_top_of(part.k);
      top[1] = finite_top_of(part.v);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      top[kv] = (unsigned)wave_max_upto((int)top[kv]);
      if ((tid & 63) == 63) sh.top[round][own][kv][tid >> 6] = top[kv];
    }
    __syncthreads();   // (one a round: the next one's maxima are in the other place)
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      top[kv] = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) top[kv] = max(top[kv], sh.top[round][own][kv][w]);
    }
    if (first + own < head1) part.store(place, top, wild, begun, codes, codes + P * D, scales);
  }
}

// A workgroup looks after `chunk` rows, and has `heads` of their heads.
template <int D, bool LIST, int HEADS>
__global__ __launch_bounds__(HEADS * kThreads) void kv_store_paged_fp8_kernel(const RowsParams p, int chunk, int heads, int Hkv) {
  __shared__ StoreShared<HEADS> sh;
  const int tid = threadIdx.x, lane = tid & 63, t = tid & (kBlock - 1);
  const int row0 = blockIdx.y * chunk, row1 = min(row0 + chunk, p.rows), head0 = blockIdx.x * heads, head1 = min(head0 + heads, Hkv);
  if (tid < kWindow) {
    const int row = row0 - (kBlock - 1) + tid, slot = row >= 0 && row < p.rows ? p.slots[row] : -1;
    sh.slot[tid] = (unsigned)slot < (unsigned)p.n_slots ? slot : -1;
  }
  __syncthreads();
  const int mine = lane < row1 - row0 ? sh.slot[kBlock - 1 + lane] : -1;   // (32 at most, the same in every wavefront)
  for (uint64_t pending = __ballot(mine >= 0); pending;) {
    const int r = __builtin_ctzll(pending), slot = __builtin_amdgcn_readlane(mine, r), slot0 = slot & -kBlock;
    pending &= ~__ballot((mine & -kBlock) == slot0);   // (-1 is in no block)
    // the row of token t, if the block's tokens stand in a row
    const int place = r + t - (slot - slot0);
    int other = sh.slot[kBlock - 1 + place] == slot0 + t ? row0 + place : -1;
    unsigned there = (unsigned)__ballot(other >= 0);
    if (there != ~0u) {
      if constexpr (LIST) {
        const int x = p.row_of[slot0 + t];
        other = (unsigned)x < (unsigned)p.rows && p.slots[x] == slot0 + t ? x : -1;   // (what no row has written is anything)
        there = (unsigned)__ballot(other >= 0);
        if (there == 0) continue;
      } else {
        __syncthreads();   // (the last block's members are not needed any more)
        if (tid < kBlock) sh.member[tid] = INT_MAX;
        __syncthreads();
        for (int i = tid; i < p.rows; i += HEADS * kThreads) {
          const unsigned off = (unsigned)p.slots[i] - (unsigned)slot0;
          if (off < (unsigned)kBlock) atomicMin(&sh.member[off], i);   // (of a slot that two rows have the first one has it)
        }
        __syncthreads();
        other = sh.member[t];
        there = (unsigned)__ballot(other != INT_MAX);
      }
    }
    const int leader = __builtin_amdgcn_readlane(other, __builtin_ctz(there));
    if (leader < row0 || leader >= row1) continue;
    __syncthreads();   // (nor its maxima)
    if (tid < kBlock) sh.member[tid] = other;
    __syncthreads();
    if (there == ~0u) store_heads<D, true, HEADS>(p, sh, there, slot0, head0, head1);
    else store_heads<D, false, HEADS>(p, sh, there, slot0, head0, head1);
  }
}

template <int D>
void launch_store(const RowsParams& p, int Hkv, bool list, hipStream_t stream) {
  // few rows: one a workgroup, one head each; more: as many of both as leave workgroups enough
  const int64_t row_heads = (int64_t)p.rows * Hkv;
  int chunk = 1;
  while (chunk < kMostChunk && row_heads / chunk > kChunkWorkgroups) chunk *= 2;
  const int64_t each = row_heads / chunk / kEnoughWorkgroups;
  const bool one = each < kHeadsAtOnce;
  const int heads = one ? 1 : (int)(each < kMostHeads ? each : kMostHeads) / kHeadsAtOnce * kHeadsAtOnce;
  const dim3 grid((unsigned)((Hkv + heads - 1) / heads), (unsigned)((p.rows + chunk - 1) / chunk)), threads((one ? 1 : kHeadsAtOnce) * kThreads);
  if (one && list) hipLaunchKernelGGL((kv_store_paged_fp8_kernel<D, true, 1>), grid, threads, 0, stream, p, chunk, heads, Hkv);
  else if (one) hipLaunchKernelGGL((kv_store_paged_fp8_kernel<D, false, 1>), grid, threads, 0, stream, p, chunk, heads, Hkv);
  else if (list) hipLaunchKernelGGL((kv_store_paged_fp8_kernel<D, true, kHeadsAtOnce>), grid, threads, 0, stream, p, chunk, heads, Hkv);
  else hipLaunchKernelGGL((kv_store_paged_fp8_kernel<D, false, kHeadsAtOnce>), grid, threads, 0, stream, p, chunk, heads, Hkv);
}

// ---------------------------------------------------------------------------------------------
// Load. Memory-bound: 8217 rows of 32 heads, D = 128 (202 MB), 36 us, 5.6 TB/s. A workgroup has 32 rows of one head. K's codes of a row are pieces of 16 channels; V's lie sixteen tokens behind one another for each
// channel, so what the rows need of V comes into LDS in such groups (rows in a row share them), and is taken from there byte by byte.
constexpr int kLoadRows = 32, kLoadGroups = 4;   // groups in LDS at a time

template <int D>
__global__ __launch_bounds__(kThreads) void kv_load_paged_fp8_kernel(const RowsParams p) {
  __shared__ alignas(16) unsigned char codes[kLoadGroups][D * kGroup];
  __shared__ int slot_of[kLoadRows], group_of[kLoadRows];   // of a row: its slot; its group's place in LDS, -1: not now, -2: a row of zeros
  constexpr int PIECES = D / 16, E = D / 32;
  const int head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, P = 1 << p.page_shift;
  for (int64_t row0 = (int64_t)blockIdx.y * kLoadRows; row0 < p.rows; row0 += (int64_t)gridDim.y * kLoadRows) {
    const int in_rows = lane & (kLoadRows - 1);
    const int slot = row0 + in_rows < p.rows ? p.slots[row0 + in_rows] : -1;
    const bool valid = (unsigned)slot < (unsigned)p.n_slots;
    if (tid < kLoadRows) slot_of[tid] = slot;
    __syncthreads();
    // K
    for (int i = tid; i < kLoadRows * PIECES; i += kThreads) {
      const int r = i / PIECES, piece = i % PIECES;
      if (row0 + r >= p.rows) break;
      const int from = slot_of[r];
      u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
      if ((unsigned)from < (unsigned)p.n_slots) {
        const char* base = head_of<D>(p, from, head);
        const int t = from & (P - 1), nth = t / kBlock;
        const u32x4 c = *reinterpret_cast<const u32x4*>(base + nth * (kBlock * D) + k_code_at(t % kBlock, piece * 16));
        const float scale = as_scale(((const unsigned char*)base)[2 * P * D + nth]);
        const u32x2 a = decode4(c[0], scale), b = decode4(c[1], scale), d = decode4(c[2], scale), e = decode4(c[3], scale);
        lo = u32x4{a[0], a[1], b[0], b[1]};
        hi = u32x4{d[0], d[1], e[0], e[1]};
      }
      u32x4* to = reinterpret_cast<u32x4*>(p.k + (row0 + r) * p.row_stride + head * p.head_stride + piece * 32);
      to[0] = lo;
      to[1] = hi;
    }
    // V: rounds of up to four groups
    uint64_t pending = __ballot(valid) & 0xffffffffu;
    bool first = true;
    do {
      int where = first && !valid && row0 + in_rows < p.rows ? -2 : -1;
      int from[kLoadGroups], n = 0;
#pragma unroll
      for (int k = 0; k < kLoadGroups; ++k) {
        from[k] = -1;
        if (pending == 0) continue;
        from[k] = __builtin_amdgcn_readlane(slot, __builtin_ctzll(pending)) & -kGroup;
        const uint64_t same = __ballot(valid && (slot & -kGroup) == from[k]) & pending;
        if ((same >> in_rows) & 1u) where = k;
        pending &= ~same;
        n = k + 1;
      }
      if (!first) __syncthreads();   // (the groups before these have been read)
      if (tid < kLoadRows) group_of[tid] = where;
      for (int i = tid; i < n * D; i += kThreads) {
        const int k = i / D, j = i % D;   // piece j of the group: row j % 32 of sum j / 32
        const int start = k == 0 ? from[0] : k == 1 ? from[1] : k == 2 ? from[2] : from[3];
        const int t = start & (P - 1), nth = t / kBlock;
        const char* base = head_of<D>(p, start, head) + P * D + nth * (kBlock * D);
        *reinterpret_cast<u32x4*>(&codes[k][j * 16]) = *reinterpret_cast<const u32x4*>(base + (((j >> 5) * 2 + ((t >> 4) & 1)) * 32 + (j & 31)) * 16);
      }
      __syncthreads();
      for (int i = tid; i < kLoadRows * (D / 8); i += kThreads) {
        const int r = i / (D / 8), c = i % (D / 8) * 8;
        const int k = group_of[r], at = slot_of[r];
        if (k == -1) continue;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (k >= 0) {
          const int t = at & (P - 1);
          const float scale = as_scale(((const unsigned char*)head_of<D>(p, at, head))[2 * P * D + kFp8VScales + t / kBlock]);
          unsigned w[2] = {0, 0};
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j >> 2] |= (unsigned)codes[k][(((c + j) % E) * 32 + (c + j) / E) * 16 + (t & 15)] << (8 * (j & 3));
          const u32x2 a = decode4(w[0], scale), b = decode4(w[1], scale);
          x = u32x4{a[0], a[1], b[0], b[1]};
        }
        *reinterpret_cast<u32x4*>(p.v + (row0 + r) * p.row_stride + head * p.head_stride + c * 2) = x;
      }
      first = false;
    } while (pending);
    __syncthreads();
  }
}

fspad_status check_rows(bool store, const fspad_paged_desc* desc, int32_t rows, const void* k, const void* v, int64_t row_stride, int64_t head_stride,
                        const int32_t* slots, const void* pages) {
  const fspad_paged_desc& d = *desc;
  if (!k || !v || !slots || !pages) return FSPAD_ERR_NULL;
  if (row_stride < 0 || head_stride < 0 || row_stride % 8 || head_stride % 8) return FSPAD_ERR_SHAPE;
  // rows and heads that overlap make no sense to write to; to read, either may be repeated
  if (!store && (head_stride < d.head_dim || row_stride < d.head_dim)) return FSPAD_ERR_SHAPE;
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)pages) & 15) return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

RowsParams rows_params(const fspad_paged_desc& d, int32_t rows, void* k, void* v, int64_t row_stride, int64_t head_stride, const int32_t* slots, void* pages) {
  RowsParams p{};
  p.k = static_cast<char*>(k); p.v = static_cast<char*>(v); p.slots = slots; p.pages = static_cast<char*>(pages);
  p.row_stride = row_stride * 2; p.head_stride = head_stride * 2; p.page_stride = d.page_stride;
  p.rows = rows; p.n_slots = d.n_pages * d.page_tokens; p.page_shift = log2_of(d.page_tokens);
  return p;
}

fspad_status check_geometry(const fspad_paged_desc* desc, int32_t rows) {
  if (!desc) return FSPAD_ERR_NULL;
  if (const fspad_status st = check_pool(*desc, PagedFormat::kFp8)) return st;
  if (rows < 0 || desc->n_kv_heads > 65535) return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

constexpr int kMaxStoreRows = 1048560;

}  // namespace

extern "C" size_t fspad_kv_page_bytes_byte(int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens) {
  if (n_kv_heads < 1 || (head_dim != 64 && head_dim != 128) || !page_tokens_ok(page_tokens, PagedFormat::kFp8)) return 0;
  return (size_t)n_kv_heads * page_head_bytes_fp8(head_dim, page_tokens);
}

extern "C" size_t fspad_kv_store_paged_byte_workspace_bytes(const fspad_paged_desc* desc, int32_t rows) {
  if (check_geometry(desc, rows) != FSPAD_OK || rows <= kScanRows) return 0;
  return (size_t)desc->n_pages * desc->page_tokens * sizeof(int32_t);
}

extern "C" fspad_status fspad_kv_store_paged_byte(const fspad_paged_desc* desc, int32_t rows, const void* k, const void* v, int64_t row_stride,
                                                 int64_t head_stride, const int32_t* slots, void* pages, void* workspace,
                                                 size_t workspace_bytes, void* hip_stream) {
  if (const fspad_status st = check_geometry(desc, rows)) return st;
  if (rows == 0) return FSPAD_OK;
  if (rows > kMaxStoreRows) return FSPAD_ERR_SHAPE;
  if (const fspad_status st = check_rows(true, desc, rows, k, v, row_stride, head_stride, slots, pages)) return st;
  const size_t need = fspad_kv_store_paged_byte_workspace_bytes(desc, rows);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return FSPAD_ERR_WORKSPACE;
  RowsParams p = rows_params(*desc, rows, const_cast<void*>(k), const_cast<void*>(v), row_stride, head_stride, slots, pages);
  p.row_of = static_cast<int32_t*>(workspace);
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (need > 0) hipLaunchKernelGGL(kv_rows_of_slots_kernel, dim3((unsigned)((rows + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p);
  if (desc->head_dim == 128) launch_store<128>(p, desc->n_kv_heads, need > 0, stream);
  else launch_store<64>(p, desc->n_kv_heads, need > 0, stream);
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}

extern "C" fspad_status fspad_kv_load_paged_byte(const fspad_paged_desc* desc, int32_t rows, const int32_t* slots, const void* pages, void* k, void* v,
                                                int64_t row_stride, int64_t head_stride, void* hip_stream) {
  if (const fspad_status st = check_geometry(desc, rows)) return st;
  if (rows == 0) return FSPAD_OK;
  if (const fspad_status st = check_rows(false, desc, rows, k, v, row_stride, head_stride, slots, pages)) return st;
  const RowsParams p = rows_params(*desc, rows, k, v, row_stride, head_stride, slots, const_cast<void*>(pages));
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const int64_t wgs = ((int64_t)rows + kLoadRows - 1) / kLoadRows;
  const dim3 grid((unsigned)desc->n_kv_heads, (unsigned)(wgs < 65535 ? wgs : 65535));
  if (desc->head_dim == 128) hipLaunchKernelGGL(kv_load_paged_fp8_kernel<128>, grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL(kv_load_paged_fp8_kernel<64>, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}
