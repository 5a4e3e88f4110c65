// Store and load of the paged 8-bit cache (include/fspad.h, "Paged 8-bit cache"). The attention over it is in fspad_attn_paged_fp8.hip. gfx950 (CDNA4) only.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"

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

// Where channel c of token t of a block lies among the block's codes.
template <int D>
__device__ __forceinline__ int k_code_at(int t, int c) { return ((c >> 4) * kBlock + t) * 16 + (c & 15); }
template <int D>
__device__ __forceinline__ int v_code_at(int t, int c) { return ((c % (D / 32) * 2 + (t >> 4)) * 32 + c / (D / 32)) * 16 + (t & 15); }

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
__device__ __forceinline__ unsigned has_wild(unsigned w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// Four channels to codes: rounded to nearest, ties to even. NaN and infinity become NaN (all bits below the sign).
__device__ __forceinline__ unsigned encode4(unsigned low, unsigned high, float scale) {
  s16x2 c = {0, 0};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, low), scale, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, high), scale, true);
  unsigned codes = __builtin_bit_cast(unsigned, c);
  if (__builtin_expect((has_wild(low) | has_wild(high)) != 0, 0)) {
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
  return encode4(x[0], x[1], scale);
}

// ---------------------------------------------------------------------------------------------
// Store. A block's scale is that of all its tokens, so one workgroup has all of a call's rows of a block (and one head): it looks for
// them, forms the largest magnitude, rounds, and where the scale of a block that holds tokens grows rounds those again. The rows of a block
// may stand anywhere in the call. Which they are is found by looking through all of a call's slots where those are few, else in a
// list by slot that a launch before this one writes; the row that has the block's lowest place leads, and its workgroup does the block.
constexpr int kScanRows = 1024;   // at most, without the list
constexpr int kChunk = 16;        // rows that a workgroup looks after, with it

__global__ __launch_bounds__(kThreads) void kv_rows_of_slots_kernel(const RowsParams p) {
  const int row = blockIdx.x * kThreads + threadIdx.x;
  if (row >= p.rows) return;
  const int slot = p.slots[row];
  if ((unsigned)slot < (unsigned)p.n_slots) p.row_of[slot] = row;
}

struct StoreShared {
  int member[kChunk][kBlock];   // row of each token of a row's block, -1: none
  unsigned there[kChunk];       // bit t: token t has one
  unsigned top[2][kThreads / 64];
  alignas(16) unsigned char codes[2][kBlock * 128];
};

// One block of one head. member: its rows; there: which tokens have one.
template <int D>
__device__ __forceinline__ void store_block(const RowsParams& p, StoreShared& sh, const int* member, unsigned there, int slot0, int head) {
  constexpr int LPR = D / 8, TOKENS = kThreads / LPR, PASSES = kBlock / TOKENS;   // lanes of a row; rows at a time
  const int P = 1 << p.page_shift, tid = threadIdx.x, part = tid % LPR;
  char* base = head_of<D>(p, slot0, head);
  const int nth = (slot0 & (P - 1)) / kBlock;
  char* codes[2] = {base + nth * (kBlock * D), base + P * D + nth * (kBlock * D)};
  unsigned char* scales[2] = {(unsigned char*)base + 2 * P * D + nth, (unsigned char*)base + 2 * P * D + kFp8VScales + nth};
  u32x4 x[PASSES][2];
  unsigned top[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int t = i * TOKENS + tid / LPR, row = member[t];
    x[i][0] = x[i][1] = u32x4{0u, 0u, 0u, 0u};
    if ((there >> t) & 1u) {
      const int64_t at = row * p.row_stride + head * p.head_stride + part * 16;
      x[i][0] = *reinterpret_cast<const u32x4*>(p.k + at);
      x[i][1] = *reinterpret_cast<const u32x4*>(p.v + at);
    }
  }
  const bool begun = there & 1u;
  int had[2] = {0, 0};
  if (!begun) {
    had[0] = *scales[0];
    had[1] = *scales[1];
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i)
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int j = 0; j < 4; ++j) top[kv] = max(top[kv], max(finite_or_zero(x[i][kv][j] & 0x7fffu), finite_or_zero((x[i][kv][j] >> 16) & 0x7fffu)));
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top[kv] = max(top[kv], (unsigned)__shfl_xor((int)top[kv], off));
    if ((tid & 63) == 0) sh.top[kv][tid >> 6] = top[kv];
  }
  __syncthreads();
  int s[2];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    unsigned all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) all = max(all, sh.top[kv][w]);
    s[kv] = max(scale_for(all), had[kv]);
    if (__builtin_expect(all > kTopBits, 0)) {
#pragma unroll
      for (int i = 0; i < PASSES; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][kv][j] = at_most_top(x[i][kv][j] & 0xffffu) | at_most_top(x[i][kv][j] >> 16) << 16;
    }
  }
  // codes of the new tokens, in the block's order
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int t = i * TOKENS + tid / LPR;
    const u32x2 kc = {encode4(x[i][0][0], x[i][0][1], as_scale(s[0])), encode4(x[i][0][2], x[i][0][3], as_scale(s[0]))};
    *reinterpret_cast<u32x2*>(&sh.codes[0][k_code_at<D>(t, part * 8)]) = kc;
    const u32x2 vc = {encode4(x[i][1][0], x[i][1][1], as_scale(s[1])), encode4(x[i][1][2], x[i][1][3], as_scale(s[1]))};
#pragma unroll
    for (int j = 0; j < 8; ++j) sh.codes[1][v_code_at<D>(t, part * 8 + j)] = (unsigned char)(vc[j >> 2] >> (8 * (j & 3)));
  }
  __syncthreads();
  // 16 bytes at a time: of K one token's, of V sixteen tokens' of one channel
  for (int i = tid; i < kBlock * D / 16; i += kThreads) {
    const int at = i * 16, t = i % kBlock, group = (i >> 5) & 1;
    u32x4* const k_to = reinterpret_cast<u32x4*>(codes[0] + at);
    if ((there >> t) & 1u) {
      *k_to = *reinterpret_cast<const u32x4*>(&sh.codes[0][at]);
    } else if (!begun && s[0] > had[0]) {
      u32x4 c = *k_to;
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = again4(c[j], as_scale(had[0]), as_scale(s[0]));
      *k_to = c;
    }
    const unsigned mine = (there >> (16 * group)) & 0xffffu;
    const bool grown = !begun && s[1] > had[1];
    if (mine || grown) {
      u32x4* const v_to = reinterpret_cast<u32x4*>(codes[1] + at);
      u32x4 c = *reinterpret_cast<const u32x4*>(&sh.codes[1][at]);
      if (mine != 0xffffu) {
        const u32x4 was = *v_to;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned bytes = (((mine >> (4 * j) & 15u) * 0x00204081u) & 0x01010101u) * 0xffu;
          c[j] = (c[j] & bytes) | ((grown ? again4(was[j], as_scale(had[1]), as_scale(s[1])) : was[j]) & ~bytes);
        }
      }
      *v_to = c;
    }
  }
  if (tid < 2 && (begun || s[tid] > had[tid])) *scales[tid] = (unsigned char)s[tid];
}

template <int D, bool SCAN>
__global__ __launch_bounds__(kThreads) void kv_store_paged_fp8_kernel(const RowsParams p) {
  __shared__ StoreShared sh;
  const int head = blockIdx.x, tid = threadIdx.x;
  if constexpr (SCAN) {   // a workgroup looks after one row
    const int row = blockIdx.y, slot = p.slots[row];
    if ((unsigned)slot >= (unsigned)p.n_slots) return;
    if (tid < kBlock) sh.member[0][tid] = INT_MAX;
    __syncthreads();
    for (int i = tid; i < p.rows; i += kThreads) {
      const unsigned off = (unsigned)p.slots[i] - (unsigned)(slot & -kBlock);
      if (off < (unsigned)kBlock) atomicMin(&sh.member[0][off], i);   // (of a slot that two rows have the first one has it)
    }
    __syncthreads();
    const unsigned there = (unsigned)__ballot(sh.member[0][tid & (kBlock - 1)] != INT_MAX);
    if (sh.member[0][__builtin_ctz(there)] != row) return;
    store_block<D>(p, sh, sh.member[0], there, slot & -kBlock, head);
  } else {
    // half a wavefront a row
    const int row0 = blockIdx.y * kChunk, t = tid & (kBlock - 1);
    for (int r = tid / kBlock; r < kChunk; r += kThreads / kBlock) {
      const int row = row0 + r, slot = row < p.rows ? p.slots[row] : -1;
      const bool valid = (unsigned)slot < (unsigned)p.n_slots;
      int other = -1;
      if (valid) {
        const int place = (slot & -kBlock) + t;
        const int x = p.row_of[place];
        if ((unsigned)x < (unsigned)p.rows && p.slots[x] == place) other = x;
      }
      unsigned there = (unsigned)(__ballot(other >= 0) >> (tid & kBlock));
      const int first = __shfl(other, (tid & kBlock) + (there ? __builtin_ctz(there) : 0));
      if (!valid || first != row) there = 0;   // (nothing to do, or another row leads)
      sh.member[r][t] = other;
      if (t == 0) sh.there[r] = there;
    }
    __syncthreads();
    for (int r = 0; r < kChunk; ++r) {
      const unsigned there = sh.there[r];
      if (there == 0) continue;
      store_block<D>(p, sh, sh.member[r], there, p.slots[row0 + r] & -kBlock, head);
      __syncthreads();   // (the codes' buffer is used again)
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Load. A workgroup has 32 rows of one head. K's codes of a row are pieces of 16 channels; V's lie sixteen tokens behind one another for each
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
        const u32x4 c = *reinterpret_cast<const u32x4*>(base + nth * (kBlock * D) + k_code_at<D>(t % kBlock, piece * 16));
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

constexpr int kMaxStoreRows = 65535 * kChunk;   // (a launch's second dimension)

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
  const unsigned heads = (unsigned)desc->n_kv_heads;
  if (need == 0) {
    const dim3 grid(heads, (unsigned)rows);
    if (desc->head_dim == 128) hipLaunchKernelGGL((kv_store_paged_fp8_kernel<128, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((kv_store_paged_fp8_kernel<64, true>), grid, dim3(kThreads), 0, stream, p);
  } else {
    hipLaunchKernelGGL(kv_rows_of_slots_kernel, dim3((unsigned)((rows + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p);
    const dim3 grid(heads, (unsigned)((rows + kChunk - 1) / kChunk));
    if (desc->head_dim == 128) hipLaunchKernelGGL((kv_store_paged_fp8_kernel<128, false>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((kv_store_paged_fp8_kernel<64, false>), grid, dim3(kThreads), 0, stream, p);
  }
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
