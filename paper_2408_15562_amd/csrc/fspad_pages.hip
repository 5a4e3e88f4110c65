// Pages that several sequences hold (include/fspad.h, "Shared pages"): forks, releases, compaction, and the copies that these leave to the
// pools. Whatever the pages' format. gfx950 (CDNA4) only.
//
// All but the copies are integers, and few: what a call costs is launches and trips to memory. So small calls are one workgroup's, which does
// one step after the other; larger ones go over the device in two or three launches, since a step that counts into `shared` or the lists has
// to be over before the next reads them.
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

constexpr int kMaxRows = 2048;          // of a block table, and forks of a call
constexpr int kMaxPages = 1 << 20;
constexpr int64_t kMaxEntries = 1 << 30;
constexpr int kAlone = 1024, kThreads = 256;   // threads of a workgroup that does a whole call, of one of several
constexpr int64_t kAloneEntries = 16384;       // table entries at most for which one does
constexpr int kAlonePages = 32768;             // and pages

__device__ __forceinline__ int page_count(int len, int page_shift, int width) {
  return (int)min(((int64_t)max(len, 0) + (1 << page_shift) - 1) >> page_shift, (int64_t)width);
}

// Sum of x over the threads before this one; over all of them in `all`. (a barrier inside; wave_sum is free again behind the next one)
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
  int32_t B, F, page_shift, n_pages, width;
};

// Who gets what: one workgroup. Lengths and the stack's height may be updated in place, so all of them are read before any is written.
__device__ void plan_forks(const ForkParams& p, int* claim, int* wave_sum) {
  constexpr int PER = kMaxRows / kAlone;
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages);
  for (int b = tid; b < p.B; b += kAlone) claim[b] = INT_MAX;
  __syncthreads();
  for (int f = tid; f < p.F; f += kAlone) {
    const unsigned d = (unsigned)p.dst[f];
    if (d < (unsigned)p.B) atomicMin(&claim[d], f);   // (the first fork that names a row has it)
  }
  __syncthreads();
  const int f0 = tid * PER;   // a thread has neighbouring forks
  int src[PER], dst[PER], n[PER], need = 0;
  bool fits[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int f = f0 + i;
    fits[i] = false;
    n[i] = 0;
    if (f >= p.F) continue;
    src[i] = p.src[f];
    dst[i] = p.dst[f];
    if ((unsigned)src[i] >= (unsigned)p.B || (unsigned)dst[i] >= (unsigned)p.B || src[i] == dst[i] || claim[dst[i]] != f) continue;
    const int have = max(p.kv_len[src[i]], 0);
    n[i] = p.n_tokens ? p.n_tokens[f] : have;
    fits[i] = p.kv_len[dst[i]] <= 0 && n[i] >= 0 && n[i] <= have && n[i] <= (int64_t)p.width << p.page_shift;
    need += fits[i] && (n[i] & ((1 << p.page_shift) - 1)) ? 1 : 0;
  }
  int all;
  int at = sum_before<kAlone>(need, wave_sum, all);   // (behind its barrier no length is read again)
  if (p.kv_len_out != p.kv_len)
    for (int b = tid; b < p.B; b += kAlone) p.kv_len_out[b] = p.kv_len[b];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int f = f0 + i;
    if (f >= p.F) continue;
    const int in_last = n[i] & ((1 << p.page_shift) - 1), full = n[i] >> p.page_shift;
    bool ok = fits[i];
    int from = -1, to = -1;
    if (ok && in_last) {
      ok = at < n_free;
      if (ok) {
        to = p.free_pages[n_free - 1 - at];
        from = p.table[src[i] * p.table_stride + full];
        p.table[dst[i] * p.table_stride + full] = to;
      }
      ++at;
    }
    const bool copied = (unsigned)from < (unsigned)p.n_pages && (unsigned)to < (unsigned)p.n_pages;
    p.copy_src[f] = copied ? from : -1;
    p.copy_dst[f] = copied ? to : -1;
    p.granted[f] = ok;
    if (ok) p.kv_len_out[dst[i]] = n[i];
  }
  if (tid == 0) *p.n_free_out = n_free - min(all, n_free);
}

// Entries of full pages, which the forks share: from the outputs of the plan.
template <int THREADS>
__device__ void share_pages(const ForkParams& p, int* before, int* wave_sum, int part, int parts) {
  constexpr int PER = kMaxRows / THREADS;
  const int tid = threadIdx.x, f0 = tid * PER;
  int sum = 0, own[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    own[i] = f0 + i < p.F && p.granted[f0 + i] ? p.kv_len_out[p.dst[f0 + i]] >> p.page_shift : 0;
    sum += own[i];
  }
  int all, at = sum_before<THREADS>(sum, wave_sum, all);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (f0 + i < p.F) before[f0 + i] = at;
    at += own[i];
  }
  __syncthreads();
  for (int x = part * THREADS + tid; x < all; x += parts * THREADS) {
    int lo = 0, hi = p.F - 1;   // the last fork with at most x entries before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] <= x) lo = mid; else hi = mid - 1;
    }
    const int i = x - before[lo], page = p.table[p.src[lo] * p.table_stride + i];
    p.table[p.dst[lo] * p.table_stride + i] = page;
    if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(&p.shared_out[page], 1);   // (sums of whole numbers: the same in any order)
  }
}

template <int THREADS>
__device__ __forceinline__ void copy_shared(const int32_t* shared, int32_t* shared_out, int n_pages, int part, int parts) {
  if (shared == shared_out) return;
  for (int i = part * THREADS + threadIdx.x; i < n_pages; i += parts * THREADS) shared_out[i] = shared[i];
}

__global__ __launch_bounds__(kAlone) void page_fork_kernel(const ForkParams p) {
  __shared__ int rows[kMaxRows], wave_sum[2][kAlone / 64];
  copy_shared<kAlone>(p.shared, p.shared_out, p.n_pages, 0, 1);
  plan_forks(p, rows, wave_sum[0]);
  __threadfence();   // (what the plan and the copy wrote to memory is read and counted in below)
  __syncthreads();
  share_pages<kAlone>(p, rows, wave_sum[1], 0, 1);
}
// the same in two launches: the first workgroup plans, the others copy
__global__ __launch_bounds__(kAlone) void page_fork_plan_kernel(const ForkParams p) {
  __shared__ int rows[kMaxRows], wave_sum[kAlone / 64];
  if (blockIdx.x == 0) plan_forks(p, rows, wave_sum);
  else copy_shared<kAlone>(p.shared, p.shared_out, p.n_pages, blockIdx.x - 1, gridDim.x - 1);
}
__global__ __launch_bounds__(kThreads) void page_fork_share_kernel(const ForkParams p) {
  __shared__ int rows[kMaxRows], wave_sum[kThreads / 64];
  share_pages<kThreads>(p, rows, wave_sum, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------------------------------
// Release. Every held entry of a sequence that ends takes one from its page's holders; a page that none is left of comes below zero, whatever the
// order, and goes onto the stack, the lowest number first.
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
  int32_t* gone;          // of several workgroups: the stack's height, then how many pages of each run of kRun go
  int64_t table_stride;
  int32_t B, page_shift, n_pages, width;
};
constexpr int kRun = 1024;   // pages

// A wavefront a row. COUNT: pages that go are counted by runs.
template <bool COUNT>
__device__ __forceinline__ void drop_rows(const ReleaseParams& p, int wave, int waves) {
  const int lane = threadIdx.x & 63;
  for (int b = wave; b < p.B; b += waves) {
    if (p.ended[b] == 0) continue;
    const int n = page_count(p.kv_len[b], p.page_shift, p.width);
    for (int i = lane; i < n; i += 64) {
      const int page = p.table[b * p.table_stride + i];
      if ((unsigned)page >= (unsigned)p.n_pages) continue;
      const int had = atomicSub(&p.shared_out[page], 1);
      if (COUNT && had == 0) atomicAdd(&p.gone[1 + page / kRun], 1);
    }
  }
}
__device__ __forceinline__ void end_rows(const ReleaseParams& p, int at, int step) {
  for (int b = at; b < p.B; b += step) p.kv_len_out[b] = p.ended[b] ? 0 : p.kv_len[b];
}

__global__ __launch_bounds__(kAlone) void page_release_kernel(const ReleaseParams p) {
  constexpr int PER = kAlonePages / kAlone;   // 32 pages a thread
  __shared__ int wave_sum[kAlone / 64];
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages);
  for (int i = tid; i < p.n_pages; i += kAlone) p.shared_out[i] = max(p.shared[i], 0);
  __threadfence();
  __syncthreads();
  drop_rows<false>(p, tid >> 6, kAlone / 64);
  __threadfence();
  __syncthreads();
  const int per = (p.n_pages + kAlone - 1) / kAlone, first = tid * per;
  unsigned gone = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int x = i < per && first + i < p.n_pages ? __hip_atomic_load(&p.shared_out[first + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    gone |= x < 0 ? 1u << i : 0u;
  }
  int all, at = n_free + sum_before<kAlone>(__builtin_popcount(gone), wave_sum, all);
  for (; gone; gone &= gone - 1) {
    const int page = first + __builtin_ctz(gone);
    if (at < p.n_pages) p.free_pages[at++] = page;
    p.shared_out[page] = 0;
  }
  end_rows(p, tid, kAlone);
  if (tid == 0) *p.n_free_out = min(n_free + all, p.n_pages);
}

__global__ __launch_bounds__(kThreads) void page_release_begin_kernel(const ReleaseParams p) {
  const int at = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
  for (int i = at; i < p.n_pages; i += step) p.shared_out[i] = max(p.shared[i], 0);
  for (int i = at; i * (int64_t)kRun < p.n_pages; i += step) p.gone[1 + i] = 0;
  if (at == 0) p.gone[0] = min(max(*p.n_free, 0), p.n_pages);
}
__global__ __launch_bounds__(kThreads) void page_release_drop_kernel(const ReleaseParams p) {
  drop_rows<true>(p, (blockIdx.x * kThreads + threadIdx.x) >> 6, gridDim.x * (kThreads / 64));
}
// A workgroup a run of pages, the last one also the lengths.
__global__ __launch_bounds__(kThreads) void page_release_push_kernel(const ReleaseParams p) {
  __shared__ int wave_sum[2][kThreads / 64];
  const int tid = threadIdx.x, runs = (p.n_pages + kRun - 1) / kRun, run = blockIdx.x;
  if (run == runs) {
    end_rows(p, tid, kThreads);
    return;
  }
  int before = 0, all;
  for (int i = tid; i < run; i += kThreads) before += p.gone[1 + i];
  const int mine = p.gone[1 + run], height = p.gone[0];
  sum_before<kThreads>(before, wave_sum[0], all);
  const int base = height + all;
  if (run == runs - 1 && tid == 0) *p.n_free_out = min(base + mine, p.n_pages);
  if (mine == 0) return;
  constexpr int PER = kRun / kThreads;
  const int first = run * kRun + tid * PER;
  unsigned gone = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) gone |= first + i < p.n_pages && p.shared_out[first + i] < 0 ? 1u << i : 0u;
  int at = base + sum_before<kThreads>(__builtin_popcount(gone), wave_sum[1], all);
  for (; gone; gone &= gone - 1) {
    const int page = first + __builtin_ctz(gone);
    if (at < p.n_pages) p.free_pages[at++] = page;
    p.shared_out[page] = 0;
  }
}

// ---------------------------------------------------------------------------------------------
// Compaction. With `keep` pages held, those that are held behind the first `keep` (movers) go to the free ones among these (holes), in order.
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
  int32_t* moved;         // workspace: how many move, the stack's height, then where page keep + i goes (itself if it does not)
  int64_t table_stride, out_stride;
  int32_t B, page_shift, n_pages, width;
};

// One workgroup: a bit of LDS for every page, ranks by sums over its words.
__global__ __launch_bounds__(kAlone) void page_compact_plan_kernel(const CompactParams p) {
  extern __shared__ unsigned bits[];   // bit of page x: it is free
  __shared__ int wave_sum[2][kAlone / 64];
  const int tid = threadIdx.x, n_free = min(max(*p.n_free, 0), p.n_pages), keep = p.n_pages - n_free, words = (p.n_pages + 31) / 32;
  for (int i = tid; i < words; i += kAlone) bits[i] = 0;
  __syncthreads();
  for (int i = tid; i < n_free; i += kAlone) {
    const unsigned page = (unsigned)p.free_pages[i];
    if (page < (unsigned)p.n_pages) atomicOr(&bits[page >> 5], 1u << (page & 31));
  }
  __syncthreads();
  // the pages of word i that lie before / from `keep` on
  auto front = [&](int i) { return keep >= 32 * i + 32 ? ~0u : keep <= 32 * i ? 0u : (1u << (keep & 31)) - 1u; };
  auto there = [&](int i) { return p.n_pages >= 32 * i + 32 ? ~0u : (1u << (p.n_pages & 31)) - 1u; };
  const int per = (words + kAlone - 1) / kAlone, w0 = tid * per, w1 = min(w0 + per, words);
  int holes = 0, movers = 0;
  for (int i = w0; i < w1; ++i) {
    holes += __builtin_popcount(bits[i] & front(i));
    movers += __builtin_popcount(~bits[i] & ~front(i) & there(i));
  }
  int all_holes, all_movers;
  int hole = sum_before<kAlone>(holes, wave_sum[0], all_holes), mover = sum_before<kAlone>(movers, wave_sum[1], all_movers);
  const int moved = min(all_holes, all_movers), most = p.n_pages / 2;   // (alike unless the stack names a page twice, or pages that are held; n_pages / 2 at most)
  for (int i = w0; i < w1; ++i) {
    for (unsigned m = bits[i] & front(i); m; m &= m - 1, ++hole)
      if (hole < moved) p.copy_dst[hole] = 32 * i + __builtin_ctz(m);
    for (unsigned m = ~bits[i] & ~front(i) & there(i); m; m &= m - 1, ++mover)
      if (mover < moved) p.copy_src[mover] = 32 * i + __builtin_ctz(m);
  }
  for (int i = moved + tid; i < most; i += kAlone) p.copy_src[i] = p.copy_dst[i] = -1;
  for (int i = tid; i < n_free; i += kAlone) p.moved[2 + i] = keep + i;
  __threadfence();   // (the lists are read back)
  __syncthreads();
  for (int k = tid; k < moved; k += kAlone) p.moved[2 + p.copy_src[k] - keep] = p.copy_dst[k];
  if (tid == 0) {
    p.moved[0] = moved;
    p.moved[1] = n_free;
  }
}

// Tables, holders and stack after the moves. Each entry is read and written by one thread: any of them may be updated in place.
__global__ __launch_bounds__(kThreads) void page_compact_apply_kernel(const CompactParams p) {
  const int moved = p.moved[0], n_free = p.moved[1], keep = p.n_pages - n_free;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
  auto place = [&](int page) { return page >= keep && page < p.n_pages ? p.moved[2 + page - keep] : page; };
  const bool tables_apart = p.table_out != p.table, holders_apart = p.shared_out != p.shared;
  for (int64_t x = at; x < (int64_t)p.B * p.width; x += step) {   // (2^30 at most)
    const int b = (int)((unsigned)x / (unsigned)p.width), i = (int)x - b * p.width;
    const bool held = i < page_count(p.kv_len[b], p.page_shift, p.width);
    if (!held && !tables_apart) continue;
    const int page = p.table[b * p.table_stride + i];
    p.table_out[b * p.out_stride + i] = held ? place(page) : page;
  }
  for (int64_t x = at; x < moved; x += step) {
    const int from = p.copy_src[x], to = p.copy_dst[x], holders = p.shared[from];
    p.shared_out[to] = holders;
    p.shared_out[from] = 0;
  }
  // (a hole is free: what it has of holders is replaced by the mover's above, and is nobody's else)
  if (holders_apart)
    for (int64_t x = at; x < p.n_pages; x += step) {
      const bool goes = x >= keep && place((int)x) != (int)x;
      bool comes = false;
      if (x < keep && moved > 0) {   // among the holes, which are in order
        int lo = 0, hi = moved - 1;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (p.copy_dst[mid] < (int)x) lo = mid + 1; else hi = mid;
        }
        comes = p.copy_dst[lo] == (int)x;
      }
      if (!goes && !comes) p.shared_out[x] = p.shared[x];
    }
  for (int64_t x = at; x < p.n_pages; x += step) p.free_out[x] = x < n_free ? p.n_pages - 1 - (int)x : -1;
}

// ---------------------------------------------------------------------------------------------
// Copies. Memory-bound: a workgroup takes 16 KB of a pair at a time.
struct CopyParams {
  char* pages;
  const int32_t* src;
  const int32_t* dst;
  int64_t page_stride;
  int32_t n_pages, n_copies, pieces, page_units;   // pieces of a page; its 16-byte units
};
constexpr int kPieceUnits = 1024;

__global__ __launch_bounds__(kThreads) void page_copy_kernel(const CopyParams p) {
  constexpr int PER = kPieceUnits / kThreads;
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
      if (at + i * kThreads < p.page_units) x[i] = a[at + i * kThreads];
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (at + i * kThreads < p.page_units) b[at + i * kThreads] = x[i];
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
unsigned workgroups(int64_t items, int64_t each, int64_t most) {
  const int64_t n = (items + each - 1) / each;
  return (unsigned)(n < 1 ? 1 : n < most ? n : most);
}

}  // namespace

extern "C" fspad_status fspad_page_fork(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int32_t n_forks,
                                        const int32_t* src, const int32_t* dst, const int32_t* n_tokens, const int32_t* kv_len,
                                        int32_t* block_table, const int32_t* free_pages, const int32_t* n_free, const int32_t* shared,
                                        int32_t* copy_src, int32_t* copy_dst, int32_t* kv_len_out, int32_t* n_free_out,
                                        int32_t* shared_out, int32_t* granted, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (n_forks < 1 || n_forks > kMaxRows) return FSPAD_ERR_SHAPE;
  if (!src || !dst || !kv_len || !block_table || !free_pages || !n_free || !shared || !copy_src || !copy_dst || !kv_len_out || !n_free_out || !shared_out || !granted)
    return FSPAD_ERR_NULL;
  const ForkParams p = {src, dst, n_tokens, kv_len, block_table, free_pages, n_free, shared, copy_src, copy_dst, kv_len_out, n_free_out, shared_out, granted,
                        table_stride, B, n_forks, log2_of(page_tokens), n_pages, table_width};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const int64_t entries = (int64_t)n_forks * table_width;
  if (entries <= kAloneEntries && (n_pages <= kAlonePages || shared == shared_out)) {
    hipLaunchKernelGGL(page_fork_kernel, dim3(1), dim3(kAlone), 0, stream, p);
  } else {
    hipLaunchKernelGGL(page_fork_plan_kernel, dim3(1 + workgroups(shared == shared_out ? 0 : n_pages, 4 * kAlone, 255)), dim3(kAlone), 0, stream, p);
    hipLaunchKernelGGL(page_fork_share_kernel, dim3(workgroups(entries, 4 * kThreads, 1024)), dim3(kThreads), 0, stream, p);
  }
  return launched();
}

extern "C" size_t fspad_page_release_workspace_bytes(int32_t B, int32_t n_pages, int32_t table_width) {
  if (check_table(B, kMinPageTokens, n_pages, table_width, table_width) != FSPAD_OK) return 0;
  if (n_pages <= kAlonePages && (int64_t)B * table_width <= kAloneEntries) return 0;
  return (size_t)(1 + (n_pages + kRun - 1) / kRun) * sizeof(int32_t);
}

extern "C" fspad_status fspad_page_release(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, const int32_t* ended,
                                           const int32_t* kv_len, const int32_t* block_table, int32_t* free_pages, const int32_t* n_free,
                                           const int32_t* shared, int32_t* kv_len_out, int32_t* n_free_out, int32_t* shared_out,
                                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (!ended || !kv_len || !block_table || !free_pages || !n_free || !shared || !kv_len_out || !n_free_out || !shared_out) return FSPAD_ERR_NULL;
  const size_t need = fspad_page_release_workspace_bytes(B, n_pages, table_width);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return FSPAD_ERR_WORKSPACE;
  const ReleaseParams p = {ended, kv_len, block_table, free_pages, n_free, shared, kv_len_out, n_free_out, shared_out, static_cast<int32_t*>(workspace), table_stride, B,
                           log2_of(page_tokens), n_pages, table_width};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (need == 0) {
    hipLaunchKernelGGL(page_release_kernel, dim3(1), dim3(kAlone), 0, stream, p);
  } else {
    const int runs = (n_pages + kRun - 1) / kRun;
    hipLaunchKernelGGL(page_release_begin_kernel, dim3(workgroups(n_pages, 4 * kThreads, 1024)), dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(page_release_drop_kernel, dim3(workgroups(B, kThreads / 64, 1024)), dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(page_release_push_kernel, dim3((unsigned)runs + 1), dim3(kThreads), 0, stream, p);
  }
  return launched();
}

extern "C" size_t fspad_page_compact_workspace_bytes(int32_t n_pages) {
  if (n_pages < 1 || n_pages > kMaxPages) return 0;
  return (size_t)(2 + (int64_t)n_pages) * sizeof(int32_t);
}

extern "C" fspad_status fspad_page_compact(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int64_t out_stride,
                                           const int32_t* kv_len, const int32_t* block_table, const int32_t* free_pages, const int32_t* n_free,
                                           const int32_t* shared, int32_t* copy_src, int32_t* copy_dst, int32_t* block_table_out,
                                           int32_t* free_out, int32_t* shared_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const fspad_status st = check_table(B, page_tokens, n_pages, table_width, table_stride)) return st;
  if (out_stride < table_width || (block_table_out == block_table && out_stride != table_stride)) return FSPAD_ERR_SHAPE;
  if (!kv_len || !block_table || !free_pages || !n_free || !shared || !block_table_out || !free_out || !shared_out) return FSPAD_ERR_NULL;
  if (n_pages > 1 && (!copy_src || !copy_dst)) return FSPAD_ERR_NULL;
  if (!workspace || workspace_bytes < fspad_page_compact_workspace_bytes(n_pages) || ((uintptr_t)workspace & 15)) return FSPAD_ERR_WORKSPACE;
  const CompactParams p = {kv_len, block_table, free_pages, n_free, shared, copy_src, copy_dst, block_table_out, free_out, shared_out,
                           static_cast<int32_t*>(workspace), table_stride, out_stride, B, log2_of(page_tokens), n_pages, table_width};
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const unsigned lds = (unsigned)((n_pages + 31) / 32 * 4);
  if (lds > 65536 && hipFuncSetAttribute(reinterpret_cast<const void*>(page_compact_plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxPages / 8) != hipSuccess)
    return FSPAD_ERR_HIP;
  hipLaunchKernelGGL(page_compact_plan_kernel, dim3(1), dim3(kAlone), lds, stream, p);
  const int64_t entries = (int64_t)B * table_width;
  hipLaunchKernelGGL(page_compact_apply_kernel, dim3(workgroups(entries > n_pages ? entries : n_pages, kThreads, 1024)), dim3(kThreads), 0, stream, p);
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
  hipLaunchKernelGGL(page_copy_kernel, dim3(workgroups((int64_t)n_copies * pieces, 1, 8192)), dim3(kThreads), 0, reinterpret_cast<hipStream_t>(hip_stream), p);
  return launched();
}
