// The page tables of a paged cache, built on the GPU: pages for new tokens from a list of free ones, and pages of ended sequences
// back on it.
//
// Both are exclusive sums over the sequences (of rows, of pages) and then one independent step for every page and every row: which sequence it
// belongs to is found by bisection in the sums.  A few KB to a few MB are moved, so what bounds a call is latency: one launch, no
// CTA waits for another.  Every CTA makes the sums of all sequences by itself (1024 at a time, a thread a sequence; a second
// pass of loads from L2 costs less than a launch or a barrier over the grid) and takes its share of the pages and rows.  The sums also
// say, before anything is written, whether the call can be done at all: it is done whole or not at all.
// Lengths and the count may be updated in place; then the CTA that ends last does that, when no other reads them any more.
#include <algorithm>

#include "cache.cuh"

namespace heart {
namespace {

constexpr int kThreads = 1024, kTableWarps = kThreads / 32;
constexpr int kWorkPerCta = 1024;  // rows or pages: one a thread, in a few CTAs as fast as in one (one sequence of 4000 new tokens 4.3 us captured, by two a thread 5.0)
constexpr int kAtOnce = 4;         // of them that a thread asks for before it stores (1024 x 900 new tokens 9.1 us, one by one 10.2; 1024 x 1000 pages given back 7.3 and 8.9)

struct TableParams {
  const int32_t *lens, *new_len;   // new_len: extend
  const uint8_t *ended;            // release
  int32_t *free_pages;
  const int32_t *free_count;
  int32_t *table, *row_start, *lens_out, *count_out;
  long long *slots;
  int32_t *status;
  unsigned *ticket;                // zero between launches
  int S, T, page_log2, n_pages, table_stride;
  bool deferred;                   // lengths or count in place, several CTAs
};

struct TableShared {
  long long sums[2][kTableWarps];
  int row[kThreads + 1], page[kThreads + 1], len[kThreads];  // of a round's sequences: rows and pages before it, tokens before the call
  int bad;
  int last;
};

// Exclusive sums of two numbers a thread over the CTA, and their totals.
__device__ __forceinline__ void scan2(TableShared &sh, long long &a, long long &b, long long &all_a, long long &all_b) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto upto_lane = [&](long long x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    return x;
  };
  const long long x = upto_lane(a), y = upto_lane(b);
  __syncthreads();
  if (lane == 31) sh.sums[0][warp] = x, sh.sums[1][warp] = y;
  __syncthreads();
  const long long u = upto_lane(sh.sums[0][lane]), v = upto_lane(sh.sums[1][lane]);
  const long long before_u = __shfl_sync(0xffffffffu, u, max(warp - 1, 0)), before_v = __shfl_sync(0xffffffffu, v, max(warp - 1, 0));
  all_a = __shfl_sync(0xffffffffu, u, 31);
  all_b = __shfl_sync(0xffffffffu, v, 31);
  a = x - a + (warp > 0 ? before_u : 0);
  b = y - b + (warp > 0 ? before_v : 0);
}

// The last i < n with at[i] <= x (at ascends, at[0] <= x).
__device__ __forceinline__ int place_of(const int *at, int n, int x) {
  int lo = 0;
  for (int step = kThreads / 2; step; step >>= 1)
    if (lo + step < n && at[lo + step] <= x) lo += step;
  return lo;
}

template <bool Extend>
__global__ void __launch_bounds__(kThreads) table_kernel(const TableParams p) {
  __shared__ TableShared sh;
  const int tid = threadIdx.x;
  if (tid == 0) sh.bad = 0;
  pdl_wait();
  pdl_launch_dependents();
  const long long most = (long long)p.table_stride << p.page_log2;
  auto pages_of = [&](long long tokens) { return (tokens + (1 << p.page_log2) - 1) >> p.page_log2; };
  // A sequence: its tokens, the rows that are new, the pages that it takes or gives back.
  auto look = [&](int s, int &len, long long &rows, long long &pages) {
    len = __ldcg(&p.lens[s]);
    rows = Extend ? __ldcg(&p.new_len[s]) : 0;
    pages = 0;
    if (!Extend && __ldcg(&p.ended[s]) == 0) return true;
    if (len < 0 || rows < 0 || len + rows > most) return false;
    pages = Extend ? pages_of(len + rows) - pages_of(len) : pages_of(len);
    return true;
  };
  // ------------------------------------------------------------------ can it be done?
  int len = 0;
  long long rows = 0, pages = 0, all_rows = 0, all_pages = 0;
  const int count = __ldcg(p.free_count);
  __syncthreads();
  for (int base = 0; base < p.S; base += kThreads) {
    int len_here = 0;
    long long rows_here = 0, pages_here = 0;
    if (base + tid < p.S && !look(base + tid, len_here, rows_here, pages_here)) {
      sh.bad = 1;
      rows_here = pages_here = 0;
    }
    if (base == 0) len = len_here, rows = rows_here, pages = pages_here;
    all_rows += rows_here;
    all_pages += pages_here;
  }
  long long total_rows, total_pages, first_row = rows, first_page = pages;
  if (p.S <= kThreads) {
    scan2(sh, first_row, first_page, total_rows, total_pages);
  } else {
    scan2(sh, all_rows, all_pages, total_rows, total_pages);
  }
  __syncthreads();
  const bool done = sh.bad == 0 && count >= 0 && count <= p.n_pages && total_rows <= p.T && total_pages <= (Extend ? count : p.n_pages - count);
  const int rows_in_use = done ? (int)total_rows : 0;
  const unsigned share = blockIdx.x * kThreads + tid, shares = gridDim.x * kThreads;
  // ------------------------------------------------------------------ the sequences, 1024 at a time
  long long row_base = 0, page_base = 0;
#pragma unroll 1
  for (int base = 0; base < p.S; base += kThreads) {
    const int s = base + tid, n = min(p.S - base, kThreads);
    long long round_rows = total_rows, round_pages = total_pages;
    if (p.S > kThreads) {
      rows = pages = 0;
      if (s < p.S && !look(s, len, rows, pages)) rows = pages = 0;
      first_row = rows, first_page = pages;
      scan2(sh, first_row, first_page, round_rows, round_pages);
    }
    if (Extend && blockIdx.x == 0 && s < p.S) p.row_start[s] = done ? (int)(row_base + first_row) : 0;
    if (!p.deferred && blockIdx.x == 0 && s < p.S) {
      if (Extend) p.lens_out[s] = done ? len + (int)rows : len;
      else p.lens_out[s] = done && __ldcg(&p.ended[s]) != 0 ? 0 : len;
    }
    if (!done) continue;
    sh.row[tid] = (int)(row_base + first_row);
    sh.page[tid] = (int)(page_base + first_page);
    sh.len[tid] = len;
    __syncthreads();
    for (unsigned first = share; first < round_pages; first += kAtOnce * shares) {
      int32_t *to[kAtOnce], page[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const unsigned i = first + j * shares;
        if (i >= round_pages) break;
        const int at = (int)page_base + (int)i, k = place_of(sh.page, n, at), place = at - sh.page[k];
        int32_t *const row = p.table + (size_t)(base + k) * p.table_stride;
        to[j] = Extend ? &row[(int)pages_of(sh.len[k]) + place] : &p.free_pages[count + at];
        page[j] = __ldcg(Extend ? &p.free_pages[count - 1 - at] : &row[place]);
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (first + j * shares < round_pages) *to[j] = page[j];
    }
    if (Extend && p.slots != nullptr) {
      for (unsigned first = share; first < round_rows; first += kAtOnce * shares) {
        long long slot[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const unsigned i = first + j * shares;
          if (i >= round_rows) break;
          const int r = (int)row_base + (int)i, k = place_of(sh.row, n, r), pos = sh.len[k] + r - sh.row[k];
          const int held = (int)pages_of(sh.len[k]), at = pos >> p.page_log2;
          // (a page that is new comes from the list: its entry of the table may be another CTA's to write)
          const int page = __ldcg(at < held ? &p.table[(size_t)(base + k) * p.table_stride + at] : &p.free_pages[count - 1 - (sh.page[k] + at - held)]);
          slot[j] = ((long long)page << p.page_log2) + (pos & ((1 << p.page_log2) - 1));
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (first + j * shares < round_rows) p.slots[(int)row_base + (int)(first + j * shares)] = slot[j];
      }
    }
    row_base += round_rows;
    page_base += round_pages;
    __syncthreads();
  }
  if (Extend && p.slots != nullptr)
    for (unsigned r = rows_in_use + share; r < (unsigned)p.T; r += shares) p.slots[r] = -1;
  const int count_after = !done ? count : Extend ? count - (int)total_pages : count + (int)total_pages;
  if (blockIdx.x == 0 && tid == 0) {
    if (Extend) p.row_start[p.S] = rows_in_use;
    if (!done) atomicExch(p.status, HEART_ERR_DEVICE_CHECK);
    if (!p.deferred) *p.count_out = count_after;
  }
  if (!p.deferred) return;
  // ------------------------------------------------------------------ in place: by the CTA that ends last
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    sh.last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    if (sh.last) *p.ticket = 0u;
    __threadfence();
  }
  __syncthreads();
  if (!sh.last) return;
  for (int s = tid; s < p.S; s += kThreads) {
    const int before = __ldcg(&p.lens[s]);
    if (Extend) p.lens_out[s] = done ? before + __ldcg(&p.new_len[s]) : before;
    else p.lens_out[s] = done && __ldcg(&p.ended[s]) != 0 ? 0 : before;
  }
  if (tid == 0) *p.count_out = count_after;
}

template <bool Extend>
cudaError_t launch(TableParams &p, const CacheGeom &g, const CacheWorkspace &w, long long work, cudaStream_t s, int *launches) {
  p.status = w.status;
  p.ticket = reinterpret_cast<unsigned *>(w.status + kTableTicketWord);
  p.S = g.S;
  p.T = g.T;
  p.page_log2 = g.page == 16 ? 4 : g.page == 32 ? 5 : g.page == 64 ? 6 : 7;
  p.n_pages = g.n_pages;
  p.table_stride = g.table_stride;
  const int ctas = (int)max(1LL, min((work + kWorkPerCta - 1) / kWorkPerCta, (long long)kCacheCtas));
  p.deferred = ctas > 1 && (p.lens == p.lens_out || p.free_count == p.count_out);
  ++*launches;
  return launch_pdl(table_kernel<Extend>, dim3(ctas), dim3(kThreads), 0, s, p);
}

}  // namespace

cudaError_t launch_cache_extend(const CacheGeom &g, const CacheWorkspace &w, const int32_t *new_len, const int32_t *kv_len, const int32_t *free_pages,
                                const int32_t *free_count, int32_t *page_table, int32_t *row_start, int32_t *kv_len_out, int32_t *free_count_out,
                                int64_t *slots, cudaStream_t s, int *launches) {
  TableParams p = {};
  p.lens = kv_len;
  p.new_len = new_len;
  p.free_pages = const_cast<int32_t *>(free_pages);
  p.free_count = free_count;
  p.table = page_table;
  p.row_start = row_start;
  p.lens_out = kv_len_out;
  p.count_out = free_count_out;
  p.slots = reinterpret_cast<long long *>(slots);
  return launch<true>(p, g, w, slots ? g.T : g.S + (long long)g.T / g.page, s, launches);
}

cudaError_t launch_cache_release(const CacheGeom &g, const CacheWorkspace &w, const uint8_t *ended, const int32_t *kv_len, int32_t *free_pages,
                                 const int32_t *free_count, const int32_t *page_table, int32_t *kv_len_out, int32_t *free_count_out, cudaStream_t s,
                                 int *launches) {
  TableParams p = {};
  p.lens = kv_len;
  p.ended = ended;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.table = const_cast<int32_t *>(page_table);
  p.lens_out = kv_len_out;
  p.count_out = free_count_out;
  return launch<false>(p, g, w, std::min((long long)g.n_pages, (long long)g.S * g.table_stride), s, launches);
}

}  // namespace heart
