// The paged 4-bit cache's own calls: quantising store, load, and the page map (block tables, slots, lengths and the stack of
// free pages from request lengths). The attention over the pages is in fspad_attn_paged.hip. gfx950 (CDNA4) only.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fspad.h"
#include "paged_layout.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// ---------------------------------------------------------------------------------------------
// Store and load. Pure data movement with a conversion: 4 bytes of bf16 K and V a channel against 17/16 of the pages, so what
// bounds a large call is memory. A lane holds 8 channels of one row (16 bytes of bf16, 4 of codes), 16 lanes a row of D = 128
// (8 of D = 64), four lanes a block. A wavefront takes neighbouring rows of ONE head: a prompt's rows are neighbours in their
// page too, so that a store instruction writes whole 256-byte stretches of codes. Workgroups that run at the same time have all heads of
// neighbouring rows, whose bf16 lies in a row: 8191 rows of 32 heads, D = 128 (170 MB), are stored and loaded in 67 us, 5.1 TB/s (41 and 26: the load finds part
// of it in the memory-side cache; 80 head after head, which reads 256 bytes in every 8 KB); 40000 rows (829 MB) in 158 us each way, 5.3 TB/s; D = 64: 80000 rows
// (829 MB) stored in 177 us and loaded in 182, 4.7 and 4.6 TB/s; 16384 rows of 8 heads, D = 128, are loaded in 14.3 us (5.9 TB/s, from that cache).
struct RowsParams {
  char* k;               // [rows] x [Hkv] x D bf16: read by the store, written by the load
  char* v;
  const int32_t* slots;
  char* pages;
  int64_t row_stride, head_stride;   // bytes
  int64_t page_stride;
  int32_t rows, n_slots, page_shift;
};

constexpr int kRowThreads = 256;

// Where a slot's codes and scales lie: addresses of this lane's 8 channels (codes), of its block (scales).
struct SlotAddr {
  char *k_code, *v_code, *k_scale, *v_scale;
};
template <int D>
__device__ __forceinline__ SlotAddr slot_addr(const RowsParams& p, int slot, int head, int part) {
  const int P = 1 << p.page_shift, t = slot & (P - 1);
  char* base = p.pages + (int64_t)(slot >> p.page_shift) * p.page_stride + (int64_t)head * page_head_bytes(D, P);
  SlotAddr a;
  a.k_code = base + t * (D / 2) + part * 4;
  // V: groups of 512/D tokens, 16 runs of D/16 channels in each, token after token in a run
  constexpr int kGroup = 512 / D, kRun = D / 32;   // tokens of a group, bytes of a run
  const int run = part * 4 / kRun;
  a.v_code = base + page_code_bytes(D, P) + ((t / kGroup) * 16 + run) * 16 + (t % kGroup) * kRun;
  a.k_scale = base + 2 * page_code_bytes(D, P) + (part / 4) * P + t;
  a.v_scale = a.k_scale + page_scale_bytes(D, P);
  return a;
}

// A block's scale byte from the bits of its largest magnitude (bf16 without the sign): the smallest s with a <= 7 * 2^(s-127).
// 7 lies halfway between the largest element and the next power of two, so no element is off by more than the scale, which is
// what rounding costs between 4 and 6 as well. 2..252 keeps every value of the block a normal, finite bf16.
__device__ __forceinline__ unsigned block_scale(unsigned top) {
  int s = (int)(top >> 7) - 2 + ((top & 0x7f) > 0x60 ? 1 : 0);
  s = min(max(s, 2), 252);
  return top >= 0x7f80u ? 255u : (unsigned)s;
}

// Largest magnitude (bits) of the four lanes' 32 channels. Magnitudes of bf16 compare as integers, NaN above infinity above the rest.
__device__ __forceinline__ unsigned block_top(const u32x4& x) {
  u16x2 m = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
  int a = max((int)m[0], (int)m[1]);
  a = max(a, __builtin_amdgcn_update_dpp(0, a, 0xB1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
  a = max(a, __builtin_amdgcn_update_dpp(0, a, 0x4E, 0xf, 0xf, true));   // quad_perm 2,3,0,1
  return (unsigned)a;
}

// Eight channels to codes. The conversion rounds to nearest, ties to even codes, and saturates at 6, of either sign.
__device__ __forceinline__ bf16x2 as_pair(unsigned w) { return __builtin_bit_cast(bf16x2, w); }   // (of a value: cast in place, an element of a vector is its first one)
__device__ __forceinline__ unsigned encode8(const u32x4& x, unsigned s) {
  const float scale = __builtin_bit_cast(float, s << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[2]), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_pair(x[3]), scale, 3);
  return s == 255u ? 0u : c;
}

// (a scale of all exponent bits makes the results NaN, for codes of zero too)
__device__ __forceinline__ u32x4 decode8(unsigned c, unsigned s) {
  const float scale = __builtin_bit_cast(float, s << 23);
  u32x4 x;
  x[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
  x[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
  x[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
  x[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  return x;
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv_store_paged_kernel(const RowsParams p) {
  constexpr int LPR = D / 8, RPW = kRowThreads / LPR;   // lanes of a row, rows of a workgroup
  const int head = blockIdx.x, part = threadIdx.x % LPR;
  for (int64_t row = (int64_t)blockIdx.y * RPW + threadIdx.x / LPR; row < p.rows; row += (int64_t)gridDim.y * RPW) {   // (whole rows: a block's four lanes stay together)
    const int slot = p.slots[row];
    if ((unsigned)slot >= (unsigned)p.n_slots) continue;
    const int64_t at = row * p.row_stride + head * p.head_stride + part * 16;
    const u32x4 kx = *reinterpret_cast<const u32x4*>(p.k + at);
    const u32x4 vx = *reinterpret_cast<const u32x4*>(p.v + at);
    const unsigned ks = block_scale(block_top(kx)), vs = block_scale(block_top(vx));
    const unsigned kc = encode8(kx, ks), vc = encode8(vx, vs);
    const SlotAddr a = slot_addr<D>(p, slot, head, part);
    *reinterpret_cast<unsigned*>(a.k_code) = kc;
    if constexpr (D == 128) {
      *reinterpret_cast<unsigned*>(a.v_code) = vc;
    } else {   // two runs of four channels, 16 bytes apart
      *reinterpret_cast<unsigned short*>(a.v_code) = (unsigned short)vc;
      *reinterpret_cast<unsigned short*>(a.v_code + 16) = (unsigned short)(vc >> 16);
    }
    if (part % 4 == 0) {
      *a.k_scale = (char)ks;
      *a.v_scale = (char)vs;
    }
  }
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void kv_load_paged_kernel(const RowsParams p) {
  constexpr int LPR = D / 8, RPW = kRowThreads / LPR;
  const int head = blockIdx.x, part = threadIdx.x % LPR;
  for (int64_t row = (int64_t)blockIdx.y * RPW + threadIdx.x / LPR; row < p.rows; row += (int64_t)gridDim.y * RPW) {
    const int slot = p.slots[row];
    u32x4 kx = {0u, 0u, 0u, 0u}, vx = {0u, 0u, 0u, 0u};
    if ((unsigned)slot < (unsigned)p.n_slots) {
      const SlotAddr a = slot_addr<D>(p, slot, head, part);
      const unsigned kc = *reinterpret_cast<const unsigned*>(a.k_code);
      unsigned vc;
      if constexpr (D == 128) vc = *reinterpret_cast<const unsigned*>(a.v_code);
      else vc = *reinterpret_cast<const unsigned short*>(a.v_code) | ((unsigned)*reinterpret_cast<const unsigned short*>(a.v_code + 16) << 16);
      kx = decode8(kc, (unsigned char)*a.k_scale);
      vx = decode8(vc, (unsigned char)*a.v_scale);
    }
    const int64_t at = row * p.row_stride + head * p.head_stride + part * 16;
    *reinterpret_cast<u32x4*>(p.k + at) = kx;
    *reinterpret_cast<u32x4*>(p.v + at) = vx;
  }
}

fspad_status move_rows(bool store, const fspad_paged_desc* desc, int32_t rows, void* k, void* v, int64_t row_stride,
                       int64_t head_stride, const int32_t* slots, void* pages, void* hip_stream) {
  if (!desc) return FSPAD_ERR_NULL;
  const fspad_paged_desc& d = *desc;
  if (const fspad_status st = check_pool(d, PagedFormat::kFp4)) return st;
  if (rows < 0 || d.n_kv_heads > 65535) return FSPAD_ERR_SHAPE;
  if (rows == 0) return FSPAD_OK;
  if (!k || !v || !slots || !pages) return FSPAD_ERR_NULL;
  if (row_stride < 0 || head_stride < 0 || row_stride % 8 || head_stride % 8) return FSPAD_ERR_SHAPE;
  // rows and heads that overlap make no sense to write to; to read, either may be repeated
  if (!store && (head_stride < d.head_dim || row_stride < d.head_dim)) return FSPAD_ERR_SHAPE;
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)pages) & 15) return FSPAD_ERR_SHAPE;
  RowsParams p{};
  p.k = static_cast<char*>(k); p.v = static_cast<char*>(v); p.slots = slots; p.pages = static_cast<char*>(pages);
  p.row_stride = row_stride * 2; p.head_stride = head_stride * 2; p.page_stride = d.page_stride;
  p.rows = rows; p.n_slots = d.n_pages * d.page_tokens; p.page_shift = log2_of(d.page_tokens);
  const int rpw = kRowThreads / (d.head_dim / 8);
  const int64_t wgs = (rows + (int64_t)rpw - 1) / rpw;
  const dim3 grid((unsigned)d.n_kv_heads, (unsigned)(wgs < 65535 ? wgs : 65535));
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (store) {
    if (d.head_dim == 128) hipLaunchKernelGGL(kv_store_paged_kernel<128>, grid, dim3(kRowThreads), 0, stream, p);
    else hipLaunchKernelGGL(kv_store_paged_kernel<64>, grid, dim3(kRowThreads), 0, stream, p);
  } else {
    if (d.head_dim == 128) hipLaunchKernelGGL(kv_load_paged_kernel<128>, grid, dim3(kRowThreads), 0, stream, p);
    else hipLaunchKernelGGL(kv_load_paged_kernel<64>, grid, dim3(kRowThreads), 0, stream, p);
  }
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}

// ---------------------------------------------------------------------------------------------
// Page map. Integers only; what a call costs is launches and trips to memory. Every workgroup reads the lengths of all
// sequences (a trip), forms the three running sums that decide everything (pages that come back, packed rows, pages that are
// needed) and then writes its share of the lists: pages pushed to the stack, new entries of the block tables, slots. None of
// these is read again: a page that is pushed and taken in one call is looked up in the table it comes from, so the workgroups
// need no order among them. Lengths and the stack's height may be updated in place, which only a workgroup that is alone, or a
// launch behind the others, can do.
struct MapParams {
  const int32_t* kv_len;
  const int32_t* n_new;
  const int32_t* path;        // may be null
  int32_t* table;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* slots;
  int32_t* kv_len_out;
  int32_t* n_free_out;
  int32_t* granted;
  int64_t table_stride;
  int32_t B, page_shift, n_pages, width, max_new, n_slots;   // max_new = 0: packed slots
};

constexpr int kMapMaxBatch = 2048;
constexpr int kMapMaxPacked = 1 << 22;
constexpr int64_t kMapMaxEntries = 1 << 30;   // of a list: indexes and one step of the grid past them stay 32-bit
// Entries (slots, and a quarter of the tables', for the pages that a call moves) that one workgroup does alone; a workgroup's share of
// more: an item a thread; workgroups at most.
constexpr int64_t kMapAlone = 4096, kMapShare = 1024, kMapMostWgs = 1024;
enum : int { kGranted = 1, kEnded = 2 };

// What a workgroup knows of every sequence (dynamic LDS, seven arrays of B words).
struct MapShared {
  int *len, *add, *have;  // length before the call, tokens asked for, pages held before the call
  int* need_before;       // pages needed by the sequences before this one
  int* back_before;       // pages that the ended sequences before this one give back
  int* row_before;        // packed rows of the sequences before this one
  int* flags;
};
constexpr int kMapArrays = 7;

// Sum of x over the threads before this one; over all of them in `all`.
template <int THREADS>
__device__ __forceinline__ int sum_before(int x, int* wave_sum, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s = wave_sum_upto(x);
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += wave_sum[w];
    all += wave_sum[w];
  }
  return before + s - x;
}

// The sequence that entry x of a list belongs to: the last one with at most x entries before it.
__device__ __forceinline__ int owner_in(const int* before, int B, int x) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (before[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <bool LISTS, bool LENGTHS, int THREADS>
__global__ __launch_bounds__(THREADS) void page_map_kernel(const MapParams p) {
  extern __shared__ int arrays[];
  __shared__ int wave_sum[3][THREADS / 64], wave_taken[THREADS / 64];
  const MapShared sh = {arrays, arrays + p.B, arrays + 2 * p.B, arrays + 3 * p.B, arrays + 4 * p.B, arrays + 5 * p.B, arrays + 6 * p.B};
  const int tid = threadIdx.x, P = 1 << p.page_shift;
  const int per = (p.B + THREADS - 1) / THREADS;   // a thread has a run of neighbouring sequences
  const int b0 = tid * per, b1 = min(b0 + per, p.B);
  const int n_free = min(max(*p.n_free, 0), p.n_pages);
  const int64_t room = (int64_t)p.width << p.page_shift;
  int back_sum = 0;
  int64_t row_sum = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = max(p.kv_len[b], 0), add = p.n_new[b];
    const int have = (int)min(((int64_t)len + P - 1) >> p.page_shift, (int64_t)p.width);
    sh.len[b] = len;
    sh.add[b] = add;
    sh.have[b] = have;
    back_sum += add < 0 ? have : 0;
    row_sum += max(add, 0);
  }
  // (rows past the end of a packed array: a share of more than the array holds counts as one more than that)
  int back_all, row_all, need_all;
  int back_at = sum_before<THREADS>(back_sum, wave_sum[0], back_all);
  int64_t row_at = sum_before<THREADS>(p.max_new > 0 ? 0 : (int)min(row_sum, (int64_t)p.n_slots + 1), wave_sum[1], row_all);
  const int avail = min(n_free + back_all, p.n_pages);
  int need_sum = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = sh.len[b], add = sh.add[b], have = sh.have[b];
    const bool ended = add < 0;
    const bool fits = !ended && (int64_t)len + add <= room && (p.max_new > 0 ? add <= p.max_new : row_at + add <= p.n_slots);
    const int need = fits ? (int)(((int64_t)len + add + P - 1) >> p.page_shift) - have : 0;
    sh.flags[b] = (ended ? kEnded : fits ? kGranted : 0);
    sh.back_before[b] = back_at;
    sh.row_before[b] = (int)min(row_at, (int64_t)p.n_slots + 1);
    sh.need_before[b] = need;
    need_sum += need;
    back_at += ended ? have : 0;
    row_at += max(add, 0);
  }
  int need_at = sum_before<THREADS>(need_sum, wave_sum[2], need_all);
  int taken = 0;
  for (int b = b0; b < b1; ++b) {
    const int need = sh.need_before[b];
    sh.need_before[b] = need_at;
    need_at += need;
    if (sh.flags[b] == kGranted) {
      if (need > 0 && need_at > avail) sh.flags[b] = 0;
      else taken = max(taken, need > 0 ? need_at : 0);
    }
  }
  __syncthreads();

  if constexpr (LISTS) {
    const int at = blockIdx.x * THREADS + tid, step = gridDim.x * THREADS;
    // entry x of the stack as the pushes leave it
    auto stacked = [&](int x) {
      if (x < n_free) return p.free_pages[x];
      const int b = owner_in(sh.back_before, p.B, x - n_free);
      return p.table[b * p.table_stride + (x - n_free - sh.back_before[b])];
    };
    // slot of token j of sequence b: in a page it has, or in one that it gets
    auto page_of = [&](int b, int i) {
      const int fresh = i - sh.have[b];
      return fresh < 0 ? p.table[b * p.table_stride + i] : stacked(avail - 1 - (sh.need_before[b] + fresh));
    };
    auto slot_in = [&](int page, int pos) {   // (an entry that names no page: no slot)
      return (unsigned)page < (unsigned)p.n_pages ? (page << p.page_shift) + (pos & (P - 1)) : -1;
    };
    // One list of everything that is written, so that the threads share it evenly whatever it is made of: pushes, entries of the
    // tables, slots four at a time
    const int pushes = back_all, entries = min(need_all, avail), total = p.max_new > 0 ? p.B * p.max_new : p.n_slots;
    const int64_t items = (int64_t)pushes + entries + (p.path ? 0 : (total + 3) / 4);
    for (int64_t item = at; item < items; item += step) {
      if (item < pushes) {
        const int x = n_free + (int)item;
        if (x < p.n_pages) p.free_pages[x] = stacked(x);
        continue;
      }
      if (item < pushes + entries) {
        const int x = (int)item - pushes, b = owner_in(sh.need_before, p.B, x);
        if (sh.flags[b] == kGranted) p.table[b * p.table_stride + sh.have[b] + (x - sh.need_before[b])] = stacked(avail - 1 - x);
        continue;
      }
      const int x0 = 4 * (int)(item - pushes - entries);
      int b = p.max_new > 0 ? x0 / p.max_new : owner_in(sh.row_before, p.B, x0), known = -1, page = -1;
      int slot[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = x0 + k;
        int first = p.max_new > 0 ? b * p.max_new : sh.row_before[b];
        // (the next sequence that has this entry; the last one has all that are left)
        while (b + 1 < p.B) {
          const int next = p.max_new > 0 ? first + p.max_new : sh.row_before[b + 1];
          if (x < next) break;
          ++b;
          first = next;
          known = -1;
        }
        const int j = x - first;
        slot[k] = -1;
        if (x < total && sh.flags[b] == kGranted && j < sh.add[b]) {
          const int pos = sh.len[b] + j, i = pos >> p.page_shift;
          if (i != known) page = page_of(b, i);
          known = i;
          slot[k] = slot_in(page, pos);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (x0 + k < total) p.slots[x0 + k] = slot[k];
    }
    if (p.path) {   // a wavefront a sequence: lane i is node i of the tree, and lane j held place j of its path
      const int lane = tid & 63;
      for (int b = at >> 6; b < p.B; b += step >> 6) {
        const int add = sh.flags[b] == kGranted ? sh.add[b] : 0;   // at most max_new <= 64
        const int node = lane < add ? p.path[(int64_t)b * p.max_new + lane] : -1;
        int place = -1;
        for (int j = add - 1; j >= 0; --j)   // (a node that is named twice has its first place)
          if (__shfl(node, j) == lane) place = j;
        if (lane < p.max_new) {
          const int pos = sh.len[b] + place;
          p.slots[(int64_t)b * p.max_new + lane] = place >= 0 ? slot_in(page_of(b, pos >> p.page_shift), pos) : -1;
        }
      }
    }
  }
  if (LENGTHS && blockIdx.x == 0) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) taken = max(taken, __shfl_xor(taken, off));
    if ((tid & 63) == 0) wave_taken[tid >> 6] = taken;
    __syncthreads();
    for (int b = tid; b < p.B; b += THREADS) {
      const int f = sh.flags[b];
      p.kv_len_out[b] = f == kEnded ? 0 : sh.len[b] + (f == kGranted ? sh.add[b] : 0);
      p.granted[b] = f == kGranted;
    }
    if (tid == 0) {
      int most = 0;
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) most = max(most, wave_taken[w]);
      *p.n_free_out = avail - most;
    }
  }
}

}  // namespace

extern "C" size_t fspad_kv_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens) {
  if (n_kv_heads < 1 || (head_dim != 64 && head_dim != 128) || !page_tokens_ok(page_tokens)) return 0;
  return (size_t)n_kv_heads * page_head_bytes(head_dim, page_tokens);
}

extern "C" fspad_status fspad_kv_store_paged(const fspad_paged_desc* desc, int32_t rows, const void* k, const void* v,
                                             int64_t row_stride, int64_t head_stride, const int32_t* slots,
                                             void* pages, void* hip_stream) {
  return move_rows(true, desc, rows, const_cast<void*>(k), const_cast<void*>(v), row_stride, head_stride, slots, pages, hip_stream);
}

extern "C" fspad_status fspad_kv_load_paged(const fspad_paged_desc* desc, int32_t rows, const int32_t* slots, const void* pages,
                                            void* k, void* v, int64_t row_stride, int64_t head_stride, void* hip_stream) {
  return move_rows(false, desc, rows, k, v, row_stride, head_stride, slots, const_cast<void*>(pages), hip_stream);
}

extern "C" fspad_status fspad_page_map(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride,
                                       const int32_t* kv_len, const int32_t* n_new, const int32_t* path, int32_t max_new,
                                       int32_t n_slots, int32_t* block_table, int32_t* free_pages, const int32_t* n_free,
                                       int32_t* slots, int32_t* kv_len_out, int32_t* n_free_out, int32_t* granted,
                                       void* hip_stream) {
  if (B < 1 || B > kMapMaxBatch || !page_tokens_ok(page_tokens) || n_pages < 1 || table_width < 1 || table_stride < table_width)
    return FSPAD_ERR_SHAPE;
  if ((int64_t)n_pages * page_tokens > INT32_MAX || (int64_t)table_width * page_tokens > INT32_MAX || (int64_t)B * table_width > kMapMaxEntries)
    return FSPAD_ERR_SHAPE;
  if (max_new < 0 || (max_new == 0 && path) || (path && max_new > FSPAD_MAX_NODES)) return FSPAD_ERR_SHAPE;
  if (max_new > 0 ? (int64_t)B * max_new > kMapMaxEntries : n_slots < 0 || n_slots > kMapMaxPacked) return FSPAD_ERR_SHAPE;
  if (!kv_len || !n_new || !block_table || !free_pages || !n_free || !kv_len_out || !n_free_out || !granted) return FSPAD_ERR_NULL;
  if (!slots && (max_new > 0 || n_slots > 0)) return FSPAD_ERR_NULL;
  MapParams p{};
  p.kv_len = kv_len; p.n_new = n_new; p.path = path; p.table = block_table; p.free_pages = free_pages; p.n_free = n_free;
  p.slots = slots; p.kv_len_out = kv_len_out; p.n_free_out = n_free_out; p.granted = granted;
  p.table_stride = table_stride;
  p.B = B; p.page_shift = log2_of(page_tokens); p.n_pages = n_pages; p.width = table_width;
  p.max_new = max_new; p.n_slots = max_new > 0 ? 0 : n_slots;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const int64_t entries = max_new > 0 ? (int64_t)B * max_new : n_slots;
  const int64_t work = entries + (int64_t)B * table_width / 4;
  const unsigned lds = (unsigned)(kMapArrays * B * sizeof(int));
  if (work <= kMapAlone) {
    hipLaunchKernelGGL((page_map_kernel<true, true, 1024>), dim3(1), dim3(1024), lds, stream, p);
  } else {
    // lengths or the stack's height in place: behind the workgroups that read them
    const bool in_place = (kv_len_out < kv_len + B && kv_len < kv_len_out + B) || n_free_out == n_free;
    int64_t wgs = (work + kMapShare - 1) / kMapShare;
    if (wgs > kMapMostWgs) wgs = kMapMostWgs;
    if (in_place) {
      hipLaunchKernelGGL((page_map_kernel<true, false, 256>), dim3((unsigned)wgs), dim3(256), lds, stream, p);
      hipLaunchKernelGGL((page_map_kernel<false, true, 256>), dim3(1), dim3(256), lds, stream, p);
    } else {
      hipLaunchKernelGGL((page_map_kernel<true, true, 256>), dim3((unsigned)wgs), dim3(256), lds, stream, p);
    }
  }
  return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP;
}
