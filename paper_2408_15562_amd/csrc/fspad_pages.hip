// Pages that several sequences hold (include/fspad.h, "Shared pages"): forks, releases, compaction, and the copies that these leave to the
// pools. Whatever the pages' format. gfx950 (CDNA4) only.
//
// All but the copies are integers, and few: what a call costs is launches and trips to memory. So workgroups find out by themselves what they have to
// know (who gets which page, where a page goes) instead of leaving it to each other in memory.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "fspad.h"
#include "paged_layout.h"
#include "wave_scan.h"

namespace {

using namespace fspad_detail;

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr int kMaxRows = 2048;          // of a block table, and forks of a call
constexpr int kMaxPages = 1 << 19;
constexpr int64_t kMaxEntries = 1 << 30;
constexpr int kThreads = 1024;
constexpr int kTile = 4096, kPer = kTile / kThreads;   // pages that a workgroup counts at a time, a thread's neighbouring ones
constexpr int kAloneTiles = 4;                         // a call on so many is one workgroup's
constexpr int kRowLanes = 16, kRowsAtOnce = kThreads / kRowLanes, kInFlight = 8;   // lanes that go along a row, rows at a time, entries that a lane asks for at once

__device__ __forceinline__ int page_count(int len, int page_shift, int width) {
  return (int)min(((int64_t)max(len, 0) + (1 << page_shift) - 1) >> page_shift, (int64_t)width);
}

// Sum of x over the threads before this one; over all of them in `all`. (a barrier inside; wave_sum is free again behind the next one)
__device__ __forceinline__ int sum_before(int x, int* wave_sum, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s = wave_sum_upto(x);
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += wave_sum[w];
    all += wave_sum[w];
  }
  return before + s - x;
}

// Calls fn(i, entry) for the first n entries of a row, from sixteen lanes of which this is one, and with an entry of -1 for some i behind them.
template <typename Fn>
__device__ __forceinline__ void along_row(const int32_t* row, int n, Fn&& fn) {
  for (int i0 = threadIdx.x % kRowLanes; i0 < n; i0 += kRowLanes * kInFlight) {
    int e[kInFlight];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) e[k] = i0 + k * kRowLanes < n ? row[i0 + k * kRowLanes] : -1;
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) fn(i0 + k * kRowLanes, e[k]);
  }
}

// How `shared` changes: a workgroup counts in LDS what happens to its own pages, for which it looks through all entries that the call is about. No
// atomics on memory: 70000 of them took 50 us (1024 rows of 31 to 250 pages, half of them released), the look takes 13, and 3.5 in a call of a few rows. What bounds it is what a compute unit
// gets from the caches, 31 bytes a ns (35 KB of entries 1.1 us; more requests out, workgroups that fetch ahead for the die, entries four at a time: the same). Eight workgroups a tile and a launch that joins them
// take 13 us for 18 there, but 12 for 9 where few of many sequences end.

// ---------------------------------------------------------------------------------------------
// Fork.
struct ForkParams {
  const int32_t* src;
  const int32_t* dst;
  const int32_t* n_tokens;    // may be null
  const int32_t* kv_len;
  int32_t* table;
  const int32_t* free_pages;
  const int32_t* n_free;
  const int32_t* shared;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* kv_len_out;
  int32_t* n_free_out;
  int32_t* shared_out;
  int32_t* granted;
  int64_t table_stride;
  int32_t B, F, page_shift, n_pages, width, tiles;   // tiles that a workgroup counts
};

// Every workgroup finds out who gets what; the first one writes it down, each copies the entries of some forks, and counts its tiles' pages. Lengths and the stack's height
// may be updated in place, which only a workgroup that is alone, or a launch behind the others, can do.
template <bool LISTS, bool LENGTHS>
__global__ __launch_bounds__(kThreads) void page_fork_kernel(const ForkParams p) {
  constexpr int PER = kMaxRows / kThreads;
  extern __shared__ int counts[];   // of the workgroup's tiles
  __shared__ int claim[kMaxRows], from_row[kMaxRows], to_row[kMaxRows], full_pages[kMaxRows], wave_sum[kThreads / 64];
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages);
  const int page0 = blockIdx.x * p.tiles * kTile, page1 = min(page0 + p.tiles * kTile, p.n_pages);   // (workgroups behind the last page count none)
  int src[PER], dst[PER], n[PER], have[PER], there[PER];
  bool rows[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {   // (a thread has neighbouring forks)
    const int f = tid * PER + i;
    src[i] = f < p.F ? p.src[f] : -1;
    dst[i] = f < p.F ? p.dst[f] : -1;
    n[i] = f < p.F && p.n_tokens ? p.n_tokens[f] : 0;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    rows[i] = (unsigned)src[i] < (unsigned)p.B && (unsigned)dst[i] < (unsigned)p.B && src[i] != dst[i];
    have[i] = rows[i] ? max(p.kv_len[src[i]], 0) : 0;
    there[i] = rows[i] ? p.kv_len[dst[i]] : 0;
  }
  for (int b = tid; b < p.B; b += kThreads) claim[b] = INT_MAX;
  for (int x = tid; x < page1 - page0; x += kThreads) counts[x] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if ((unsigned)dst[i] < (unsigned)p.B) atomicMin(&claim[dst[i]], tid * PER + i);   // (the first fork that names a row has it)
  __syncthreads();
  const int in_page = (1 << p.page_shift) - 1;
  int need = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (!p.n_tokens) n[i] = have[i];
    rows[i] = rows[i] && claim[dst[i]] == tid * PER + i && there[i] <= 0 && n[i] >= 0 && n[i] <= have[i] && n[i] <= (int64_t)p.width << p.page_shift;
    need += rows[i] && (n[i] & in_page) ? 1 : 0;
  }
  int all, at = sum_before(need, wave_sum, all);
  const bool writes = blockIdx.x == 0;
  if (LENGTHS && writes && p.kv_len_out != p.kv_len)
    for (int b = tid; b < p.B; b += kThreads) p.kv_len_out[b] = p.kv_len[b];
  if (LENGTHS && p.kv_len_out != p.kv_len) __syncthreads();   // (the forks' own are written behind them)
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int f = tid * PER + i;
    if (f >= p.F) continue;
    const bool part = rows[i] && (n[i] & in_page);
    const bool ok = rows[i] && (!part || at < n_free);
    const int full = n[i] >> p.page_shift;
    if (LISTS && writes) {
      int from = -1, to = -1;
      if (part && ok) {
        to = p.free_pages[n_free - 1 - at];
        from = p.table[src[i] * p.table_stride + full];
        p.table[dst[i] * p.table_stride + full] = to;
      }
      const bool copied = (unsigned)from < (unsigned)p.n_pages && (unsigned)to < (unsigned)p.n_pages;
      p.copy_src[f] = copied ? from : -1;
      p.copy_dst[f] = copied ? to : -1;
      p.granted[f] = ok;
    }
    if (LENGTHS && writes && ok) p.kv_len_out[dst[i]] = n[i];
    at += part ? 1 : 0;
    from_row[f] = src[i];
    to_row[f] = dst[i];
    full_pages[f] = ok ? full : 0;
  }
  if (LENGTHS && writes && tid == 0) *p.n_free_out = n_free - min(all, n_free);
  if constexpr (!LISTS) return;
  __syncthreads();
  // full pages, which both rows hold
  for (int f = tid / kRowLanes; f < p.F; f += kRowsAtOnce) {
    const int n_full = full_pages[f];
    const bool own = f % gridDim.x == blockIdx.x;
    if (n_full == 0 || !(own || page0 < page1)) continue;
    int32_t* const to = p.table + to_row[f] * p.table_stride;
    along_row(p.table + from_row[f] * p.table_stride, n_full, [&](int i, int page) {
      if (i >= n_full) return;
      if (own) to[i] = page;
      if (page >= page0 && page < page1) atomicAdd(&counts[page - page0], 1);
    });
  }
  __syncthreads();
  for (int x = page0 + tid; x < page1; x += kThreads) {
    const int more = counts[x - page0];
    if (more || p.shared_out != p.shared) p.shared_out[x] = max(p.shared[x], 0) + more;
  }
}

// ---------------------------------------------------------------------------------------------
// Release. Every held entry of a sequence that ends takes one from its page's holders; pages that none is left of go onto the stack, the lowest number first.
struct ReleaseParams {
  const int32_t* ended;
  const int32_t* kv_len;
  const int32_t* table;
  int32_t* free_pages;
  const int32_t* n_free;
  const int32_t* shared;
  int32_t* kv_len_out;
  int32_t* n_free_out;
  int32_t* shared_out;
  int32_t* gone;          // of several workgroups: the stack's height, then how many pages of each tile go
  int64_t table_stride;
  int32_t B, page_shift, n_pages, width, tiles;
};

__device__ __forceinline__ void end_rows(const ReleaseParams& p) {
  for (int b = threadIdx.x; b < p.B; b += kThreads) p.kv_len_out[b] = p.ended[b] ? 0 : p.kv_len[b];
}

// ALONE: one workgroup has all tiles, and pushes. Else each has one, and leaves a count below zero for pages that go.
template <bool ALONE>
__global__ __launch_bounds__(kThreads) void page_release_kernel(const ReleaseParams p) {
  extern __shared__ int counts[];
  __shared__ int row[kMaxRows], held[kMaxRows], n_rows, wave_sum[kAloneTiles][kThreads / 64];
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages);
  const int page0 = ALONE ? 0 : blockIdx.x * kTile, page1 = ALONE ? p.n_pages : min(page0 + kTile, p.n_pages);
  if (tid == 0) n_rows = 0;
  for (int x = tid; x < page1 - page0; x += kThreads) counts[x] = 0;
  __syncthreads();
  for (int b = tid; b < p.B; b += kThreads) {
    const int ended = p.ended[b], n = page_count(p.kv_len[b], p.page_shift, p.width);
    if (ended == 0 || n == 0) continue;
    const int at = atomicAdd(&n_rows, 1);   // (in any order: they are counted)
    row[at] = b;
    held[at] = n;
  }
  __syncthreads();
  for (int r = tid / kRowLanes; r < n_rows; r += kRowsAtOnce)
    along_row(p.table + row[r] * p.table_stride, held[r], [&](int, int page) {
      const unsigned x = (unsigned)page - page0;
      if (x < (unsigned)(page1 - page0)) atomicAdd(&counts[x], 1);
    });
  __syncthreads();
  int height = n_free;
#pragma unroll
  for (int tile = 0; tile < (ALONE ? kAloneTiles : 1); ++tile) {
    const int first = page0 + tile * kTile + tid * kPer;
    if (ALONE && tile >= p.tiles) break;
    unsigned gone = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (first + i >= page1) continue;
      const int had = p.shared[first + i], left = max(had, 0) - counts[first + i - page0];
      if (left < 0) gone |= 1u << i;
      const int now = ALONE ? max(left, 0) : max(left, -1);
      if (now != had || p.shared_out != p.shared) p.shared_out[first + i] = now;
    }
    int all, at = height + sum_before(__builtin_popcount(gone), wave_sum[tile], all);
    if (ALONE) {
      for (; gone; gone &= gone - 1, ++at)
        if (at < p.n_pages) p.free_pages[at] = first + __builtin_ctz(gone);
      height = min(height + all, p.n_pages);
    } else if (tid == 0) {
      p.gone[1 + blockIdx.x] = all;
      if (blockIdx.x == 0) p.gone[0] = n_free;
    }
  }
  if (ALONE) {
    end_rows(p);
    if (tid == 0) *p.n_free_out = height;
  }
}

// A workgroup a tile, the last one the lengths.
__global__ __launch_bounds__(kThreads) void page_release_push_kernel(const ReleaseParams p) {
  __shared__ int wave_sum[2][kThreads / 64];
  const int tid = threadIdx.x, tile = blockIdx.x;
  if (tile == p.tiles) {
    end_rows(p);
    return;
  }
  const int first = tile * kTile + tid * kPer, mine = p.gone[1 + tile], height = p.gone[0];
  unsigned gone = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) gone |= first + i < p.n_pages && p.shared_out[first + i] < 0 ? 1u << i : 0u;
  int before = 0, all;
  for (int i = tid; i < tile; i += kThreads) before += p.gone[1 + i];
  sum_before(before, wave_sum[0], all);
  const int base = height + all;
  if (tile == p.tiles - 1 && tid == 0) *p.n_free_out = min(base + mine, p.n_pages);
  int at = base + sum_before(__builtin_popcount(gone), wave_sum[1], all);
  for (; gone; gone &= gone - 1, ++at) {
    const int page = first + __builtin_ctz(gone);
    if (at < p.n_pages) p.free_pages[at] = page;
    p.shared_out[page] = 0;
  }
}

// ---------------------------------------------------------------------------------------------
// Compaction. With `keep` pages held, those that are held behind the first `keep` (movers) go to the free ones among these (holes), in order. Every workgroup
// has a bit in LDS for every page and the number of holes, and of movers, before each word of them: where a page goes is found from these, so that tables, holders and lists are
// written in one launch. (The stack, if it is updated in place, by another one.)
struct CompactParams {
  const int32_t* kv_len;
  const int32_t* table;
  const int32_t* free_pages;
  const int32_t* n_free;
  const int32_t* shared;
  int32_t* copy_src;      // [n_pages / 2]
  int32_t* copy_dst;
  int32_t* table_out;
  int32_t* free_out;
  int32_t* shared_out;
  int64_t table_stride, out_stride;
  int32_t B, page_shift, n_pages, width, words;
};

__device__ __forceinline__ void new_stack(const CompactParams& p, int n_free) {
  for (int x = blockIdx.x * kThreads + threadIdx.x; x < p.n_pages; x += gridDim.x * kThreads) p.free_out[x] = x < n_free ? p.n_pages - 1 - x : -1;
}

// The place of set bit k of a word that has as many.
__device__ __forceinline__ int nth_bit(unsigned word, int k) {
  int at = 0;
#pragma unroll
  for (int half = 16; half > 0; half >>= 1) {
    const int low = __builtin_popcount((word >> at) & ((1u << half) - 1u));
    if (k >= low) {
      k -= low;
      at += half;
    }
  }
  return at;
}

template <bool STACK>
__global__ __launch_bounds__(kThreads) void page_compact_kernel(const CompactParams p) {
  extern __shared__ unsigned bits[];       // bit of page x: it is free; behind them, the holes (or movers) before each word
  int* const before = reinterpret_cast<int*>(bits + p.words);
  __shared__ int wave_sum[2][kThreads / 64];
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages), keep = p.n_pages - n_free, border = keep >> 5;   // (the word that has both)
  for (int i = tid; i < p.words; i += kThreads) bits[i] = 0;
  __syncthreads();
  for (int i = tid; i < n_free; i += kThreads) {
    const unsigned page = (unsigned)p.free_pages[i];
    if (page < (unsigned)p.n_pages) atomicOr(&bits[page >> 5], 1u << (page & 31));
  }
  __syncthreads();
  // holes of word i; movers of it
  auto front = [&](int i) { return i < border ? ~0u : i > border ? 0u : (1u << (keep & 31)) - 1u; };
  auto holes_of = [&](int i) { return bits[i] & front(i); };
  auto movers_of = [&](int i) { return ~bits[i] & ~front(i) & (p.n_pages >= 32 * i + 32 ? ~0u : (1u << (p.n_pages & 31)) - 1u); };
  const int per = (p.words + kThreads - 1) / kThreads, w0 = min(tid * per, p.words), w1 = min(w0 + per, p.words);
  int holes = 0, movers = 0;
  for (int i = w0; i < w1; ++i) {
    holes += __builtin_popcount(holes_of(i));
    movers += __builtin_popcount(movers_of(i));
  }
  int all_holes, all_movers;
  int hole = sum_before(holes, wave_sum[0], all_holes), mover = sum_before(movers, wave_sum[1], all_movers);
  const int moved = min(all_holes, all_movers), most = p.n_pages / 2;   // (alike, if the stack is in order)
  for (int i = w0; i < w1; ++i) {
    if (i <= border) before[i] = hole;     // (of the border's word, both: its movers are the first ones)
    else before[i] = mover;
    hole += __builtin_popcount(holes_of(i));
    mover += __builtin_popcount(movers_of(i));
  }
  __syncthreads();
  // the page that hole k is, by halving; the place of a mover among the movers
  auto nth_hole = [&](int k) {
    int lo = 0, hi = min(border, p.words - 1);
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] <= k) lo = mid; else hi = mid - 1;
    }
    return 32 * lo + nth_bit(holes_of(lo), k - before[lo]);
  };
  auto rank = [&](int page) {
    const int i = page >> 5;
    return (i == border ? 0 : before[i]) + __builtin_popcount(movers_of(i) & ((1u << (page & 31)) - 1u));
  };
  auto moves = [&](int page) { return page >= keep && page < p.n_pages && !((bits[page >> 5] >> (page & 31)) & 1u) && rank(page) < moved; };
  const bool tables_apart = p.table_out != p.table, holders_apart = p.shared_out != p.shared;
  const int at = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  for (int x = at; x < p.B * p.width; x += step) {   // (2^30 at most)
    const int b = (int)((unsigned)x / (unsigned)p.width), i = x - b * p.width;
    const bool held = i < page_count(p.kv_len[b], p.page_shift, p.width);
    if (!held && !tables_apart) continue;
    const int page = p.table[b * p.table_stride + i];
    p.table_out[b * p.out_stride + i] = held && moves(page) ? nth_hole(rank(page)) : page;
  }
  for (int x = at; x < p.n_pages; x += step) {
    const bool free = (bits[x >> 5] >> (x & 31)) & 1u;
    if (moves(x)) {
      const int k = rank(x), to = nth_hole(k), holders = p.shared[x];
      p.copy_src[k] = x;
      p.copy_dst[k] = to;
      p.shared_out[to] = holders;   // (what the hole had of holders is nobody's)
      p.shared_out[x] = 0;
    } else if (holders_apart && !(free && x < keep && before[x >> 5] + __builtin_popcount(holes_of(x >> 5) & ((1u << (x & 31)) - 1u)) < moved)) {
      p.shared_out[x] = p.shared[x];
    }
  }
  for (int i = at; i < most; i += step)
    if (i >= moved) p.copy_src[i] = p.copy_dst[i] = -1;
  if (STACK) new_stack(p, n_free);
}
__global__ __launch_bounds__(kThreads) void page_compact_stack_kernel(const CompactParams p) { new_stack(p, min(max(*p.n_free, 0), p.n_pages)); }

// ---------------------------------------------------------------------------------------------
// Copies. Memory-bound: a workgroup takes 16 KB of a pair at a time. 910 pages of 131 KB (240 MB read and written) in 47 us, 5.1 TB/s.
struct CopyParams {
  char* pages;
  const int32_t* src;
  const int32_t* dst;
  int64_t page_stride;
  int32_t n_pages, n_copies, pieces, page_units;   // pieces of a page; its 16-byte units
};
constexpr int kPieceUnits = 1024, kCopyThreads = 256;

__global__ __launch_bounds__(kCopyThreads) void page_copy_kernel(const CopyParams p) {
  constexpr int PER = kPieceUnits / kCopyThreads;
  const int64_t items = (int64_t)p.n_copies * p.pieces;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int pair = (int)(item / p.pieces), piece = (int)(item - (int64_t)pair * p.pieces);
    const int from = p.src[pair], to = p.dst[pair];
    if ((unsigned)from >= (unsigned)p.n_pages || (unsigned)to >= (unsigned)p.n_pages || from == to) continue;
    const u32x4* a = reinterpret_cast<const u32x4*>(p.pages + from * p.page_stride);
    u32x4* b = reinterpret_cast<u32x4*>(p.pages + to * p.page_stride);
    const int at = piece * kPieceUnits + threadIdx.x;
    u32x4 x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (at + i * kCopyThreads < p.page_units) x[i] = a[at + i * kCopyThreads];
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (at + i * kCopyThreads < p.page_units) b[at + i * kCopyThreads] = x[i];
  }
}

fspad_status check_table(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride) {
  if (B < 1 || B > kMaxRows || !page_tokens_ok(page_tokens) || n_pages < 1 || n_pages > kMaxPages || table_width < 1 || table_stride < table_width)
    return FSPAD_ERR_SHAPE;
  if ((int64_t)n_pages * page_tokens > INT32_MAX || (int64_t)table_width * page_tokens > INT32_MAX || (int64_t)B * table_width > kMaxEntries)
    return FSPAD_ERR_SHAPE;
  return FSPAD_OK;
}

fspad_status launched() { return hipGetLastError() == hipSuccess ? FSPAD_OK : FSPAD_ERR_HIP; }
int workgroups(int64_t items, int64_t each, int64_t most) {
  const int64_t n = (items + each - 1) / each;
  return (int)(n < 1 ? 1 : n < most ? n : most);
}

}  // namespace

extern "C" fspad_status fspad_page_fork(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int32_t n_forks,
                                        const int32_t* src, const int32_t* dst, const int32_t* n_tokens, const int32_t* kv_len,
                                        int32_t* block_table, const int32_t* free_pages, const int32_t* n_free, const int32_t* shared,
                                        int32_t* copy_src, int32_t* copy_dst, int32_t* kv_len_out, int32_t* n_free_out,
                                        int32_t* shared_out, int32_t* granted, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (n_forks < 0 || n_forks > kMaxRows) return FSPAD_ERR_SHAPE;
  if (!kv_len || !block_table || !free_pages || !n_free || !shared || !kv_len_out || !n_free_out || !shared_out) return FSPAD_ERR_NULL;
  if (n_forks > 0 && (!src || !dst || !copy_src || !copy_dst || !granted)) return FSPAD_ERR_NULL;
  const int tiles = (n_pages + kTile - 1) / kTile;
  // a workgroup for every tile, and for some sixteen thousand entries that forks may copy
  const bool alone = tiles <= kAloneTiles && (int64_t)n_forks * table_width <= 4 * kTile;
  const unsigned wgs = alone ? 1u : (unsigned)std::max(tiles, workgroups((int64_t)n_forks * table_width, 4 * kTile, 256));
  const ForkParams p = {src, dst, n_tokens, kv_len, block_table, free_pages, n_free, shared, copy_src, copy_dst, kv_len_out, n_free_out, shared_out, granted,
                        table_stride, B, n_forks, log2_of(page_tokens), n_pages, table_width, alone ? tiles : 1};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const unsigned lds = (unsigned)((n_pages < p.tiles * kTile ? n_pages : p.tiles * kTile) * sizeof(int));
  if (alone || (kv_len_out != kv_len && n_free_out != n_free)) {
    hipLaunchKernelGGL((page_fork_kernel<true, true>), dim3(wgs), dim3(kThreads), lds, stream, p);
  } else {
    hipLaunchKernelGGL((page_fork_kernel<true, false>), dim3(wgs), dim3(kThreads), lds, stream, p);
    hipLaunchKernelGGL((page_fork_kernel<false, true>), dim3(1), dim3(kThreads), lds, stream, p);
  }
  return launched();
}

extern "C" size_t fspad_page_release_workspace_bytes(int32_t B, int32_t n_pages, int32_t table_width) {
  if (check_table(B, kMinPageTokens, n_pages, table_width, table_width) != FSPAD_OK) return 0;
  const int tiles = (n_pages + kTile - 1) / kTile;
  return tiles <= kAloneTiles ? 0 : (size_t)(1 + tiles) * sizeof(int32_t);
}

extern "C" fspad_status fspad_page_release(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, const int32_t* ended,
                                           const int32_t* kv_len, const int32_t* block_table, int32_t* free_pages, const int32_t* n_free,
                                           const int32_t* shared, int32_t* kv_len_out, int32_t* n_free_out, int32_t* shared_out,
                                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (!ended || !kv_len || !block_table || !free_pages || !n_free || !shared || !kv_len_out || !n_free_out || !shared_out) return FSPAD_ERR_NULL;
  const size_t need = fspad_page_release_workspace_bytes(B, n_pages, table_width);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return FSPAD_ERR_WORKSPACE;
  const int tiles = (n_pages + kTile - 1) / kTile;
  const ReleaseParams p = {ended, kv_len, block_table, free_pages, n_free, shared, kv_len_out, n_free_out, shared_out, static_cast<int32_t*>(workspace), table_stride, B,
                           log2_of(page_tokens), n_pages, table_width, tiles};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (need == 0) {
    hipLaunchKernelGGL(page_release_kernel<true>, dim3(1), dim3(kThreads), n_pages * sizeof(int), stream, p);
  } else {
    hipLaunchKernelGGL(page_release_kernel<false>, dim3((unsigned)tiles), dim3(kThreads), kTile * sizeof(int), stream, p);
    hipLaunchKernelGGL(page_release_push_kernel, dim3((unsigned)tiles + 1), dim3(kThreads), 0, stream, p);
  }
  return launched();
}

extern "C" fspad_status fspad_page_compact(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int64_t out_stride,
                                           const int32_t* kv_len, const int32_t* block_table, const int32_t* free_pages, const int32_t* n_free,
                                           const int32_t* shared, int32_t* copy_src, int32_t* copy_dst, int32_t* block_table_out,
                                           int32_t* free_out, int32_t* shared_out, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (out_stride < table_width || (block_table_out == block_table && out_stride != table_stride)) return FSPAD_ERR_SHAPE;
  if (!kv_len || !block_table || !free_pages || !n_free || !shared || !block_table_out || !free_out || !shared_out) return FSPAD_ERR_NULL;
  if (n_pages > 1 && (!copy_src || !copy_dst)) return FSPAD_ERR_NULL;
  const int words = (n_pages + 31) / 32;
  const CompactParams p = {kv_len, block_table, free_pages, n_free, shared, copy_src, copy_dst, block_table_out, free_out, shared_out, table_stride, out_stride, B,
                           log2_of(page_tokens), n_pages, table_width, words};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const unsigned lds = (unsigned)(2 * words * sizeof(int));
  const int64_t entries = (int64_t)B * table_width;
  const unsigned wgs = (unsigned)workgroups(entries > n_pages ? entries : n_pages, kThreads, 256);
  if (free_out != free_pages || wgs == 1) {
    hipLaunchKernelGGL(page_compact_kernel<true>, dim3(wgs), dim3(kThreads), lds, stream, p);
  } else {
    hipLaunchKernelGGL(page_compact_kernel<false>, dim3(wgs), dim3(kThreads), lds, stream, p);
    hipLaunchKernelGGL(page_compact_stack_kernel, dim3((unsigned)workgroups(n_pages, 4 * kThreads, 256)), dim3(kThreads), 0, stream, p);
  }
  return launched();
}

extern "C" fspad_status fspad_page_copy(void* pages, int32_t n_pages, int64_t page_stride, int64_t page_bytes, int32_t n_copies, const int32_t* copy_src,
                                        const int32_t* copy_dst, void* hip_stream) {
  if (n_pages < 1 || page_bytes < 16 || page_bytes % 16 || page_bytes > INT32_MAX || page_stride < page_bytes || page_stride % 16 || page_stride > UINT32_MAX || n_copies < 0)
    return FSPAD_ERR_SHAPE;
  if (n_copies == 0) return FSPAD_OK;
  if (!pages || !copy_src || !copy_dst) return FSPAD_ERR_NULL;
  if ((uintptr_t)pages & 15) return FSPAD_ERR_SHAPE;
  const int units = (int)(page_bytes / 16), pieces = (units + kPieceUnits - 1) / kPieceUnits;
  const CopyParams p = {static_cast<char*>(pages), copy_src, copy_dst, page_stride, n_pages, n_copies, pieces, units};
  hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)workgroups((int64_t)n_copies * pieces, 1, 8192)), dim3(kCopyThreads), 0, reinterpret_cast<hipStream_t>(hip_stream), p);
  return launched();
}
