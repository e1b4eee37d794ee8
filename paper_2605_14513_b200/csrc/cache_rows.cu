// Attention over a paged cache for few query rows a sequence and key head: single tokens and drafted tokens.
//
// Every key and value is read once and used by 8 or 16 rows, so HBM bounds it: a step of 128 keys is 64 KB, 2800 clocks of an SM's share of
// the bandwidth (1400 as e4m3), and its products take 256 clocks of the warp-wide matrix instruction for every 8 rows.  So the design is
// about bytes in flight: one CTA an SM, eight warps, each with a ring of its own of 24 KB that tensor copies fill.  A warp takes 16 of
// every 128 keys (32 of 256 where they are e4m3), with the running maximum and sum of its own keys, so nothing but the warp's own barrier is
// waited for until a tile's end.  Keys and values are the first operands of the products, rows the second: a product has 16 of the former and 8 of
// the latter, and most calls have no more rows.  (Rows first, 16 of them: 20 x 8001 tokens e4m3, 32 heads on 8, 91 us against 75; 12 warps with
// smaller rings 74, and one token over 4k 11.5 us instead of 10.8.)
//
// With eight warps an SM what comes next are instructions: 900 for 16 keys, converting keys and values from e4m3 to bf16, took 4700 clocks.
// The conversion to f16 is one instruction for two codes, so e4m3 caches are multiplied in f16, which holds codes exactly:
//   * a query row, scaled by a power of two to a largest element in [2^14, 2^15), is in f16 what it is in bf16 (but for elements below
//     2^-32 of the largest, which lose bits);
//   * values are the codes; a token's scale 2^e goes into its weight, behind the mask, so that what a row does not see has no part in it: the product takes
//     2^(score + e - m), between 0 and 2^14, the row's largest so far at 2^6 to 2^14.  One below 2^-31 of it counts as zero.
//   * the row sum, of 2^(score - m'), has a reference of its own, a lane's: scales may be any number of binades apart.  (Eight exponentials more for 32
//     keys, and no multiplication of values: 64 single tokens over up to 16k, 32 heads on 8, 251 us, and as long with the scales multiplied into values.)
// (The warp-wide products of e4m3 codes themselves are carried out as conversions and f16 products here, 96 for the 64 in the source.)
//
// Work: rows of a sequence and key head, packed as (token, query head of the group), in tiles of 8 or 16; all key steps of all tiles in one line,
// (sequence, head, tile, step), are cut into equal shares, one a CTA; what a CTA has of a tile that it does not have whole goes to the
// workspace, and the CTA that brings the last part puts the tile together, its parts in order: the result does not depend on which
// one came last.  Every CTA finds its share by itself from the sequences' lengths, so the launch needs no plan and no lengths on the host, and a
// captured one follows the lengths.
//
// Behind the tile kernel of an e4m3 cache the same code does those sequences and key heads again whose scales that kernel cannot hold, whole tiles
// of 16 rows dealt in turn; as a rule there are none, and the launch ends at once.
#include <cuda.h>

#include "cache.cuh"
#include "tc_ptx.cuh"

namespace heart {
using namespace tc;
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRing = 24576;           // bytes a warp
constexpr int kMaxStages = 3;
constexpr int kMaxParts = 31;          // of a tile, and one more where shares cross tiles: the last CTA reads them, a lane a part
constexpr int kApartRows = 6;          // rows of a tile whose sums have a place beside the rings
constexpr float kNoReference = -3.0e38f;
constexpr float kMaxGrowth = 8.f;      // log2: the reference of a row moves when a maximum exceeds it by more
constexpr float kHeadroomE4m3 = 6.f;   // log2 of the largest weight when the reference has moved

struct True {
  static constexpr bool value = true;
};
struct False {
  static constexpr bool value = false;
};

struct RowsParams {
  CacheIndex ix;
  const uint16_t *Q;
  uint16_t *O;
  float *lse;
  const uint8_t *k_scale, *v_scale;
  long long qt, qh;
  int Hq, Hkv, G;
  float scale_log2;
  int test_skip;  // test-hook builds only: the first warp of CTA 0 leaves out its second copy
  int32_t *arrivals;
  float *parts;
  float2 *part_l;
  const uint8_t *redo;   // see CacheWorkspace
  const int *any_redo;
  int looked;
};

struct alignas(16) RowsShared {
  uint64_t full[kWarps][kMaxStages];
  alignas(16) uint8_t scales[kWarps][kMaxStages][64];  // e4m3: of the keys and of the values of a stage
  float2 l[kWarps][16];   // row sums and their references
  float o_ref[kWarps][16];  // e4m3: references of the sums of values
  long long total[kWarps];
  int longest[kWarps];
  int found;              // sequence of the CTA's first step
  int found_q[3];
  long long found_at, found_steps;  // steps before it, and of one of its heads
  int last;
  int abort;
};
constexpr int kRowsSmem = kWarps * kRing + sizeof(RowsShared) + kWarps * kApartRows * 512;
static_assert(kRowsSmem <= 232448 && sizeof(RowsShared) % 16 == 0, "shared memory of an SM");

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, int bytes, uint64_t *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ bool not_finite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }
// Of four codes, the top bits of those that are no numbers, 0x7f or 0xff (and other bits).
__device__ __forceinline__ uint32_t ends_of(uint32_t codes) { return (codes & 0x7f7f7f7fu) + 0x01010101u; }

// The 8 x 8 matrix of 16-bit numbers that the warp holds, a row to four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// Scale bytes of tokens that there are not: the smallest, so that their values of zero raise no row's reference.
__device__ alignas(16) const uint8_t kNoScales[32] = {};

// Keys that a warp takes at a time, 4 KB of them.
__host__ __device__ constexpr int keys_of(bool e4m3) { return e4m3 ? 32 : 16; }

template <int NT, bool E4m3, bool Redo>
__global__ void __launch_bounds__(kThreads, 1)
    cache_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const RowsParams p) {
  constexpr int kRows = 8 * NT;
  constexpr int kKeys = keys_of(E4m3), kStep = kWarps * kKeys, kTiles = kKeys / 16;  // keys a warp takes at a time, a step, products of 16 keys
  constexpr int kKeysLog2 = kKeys == 32 ? 5 : 4;
  constexpr int kHalf = kKeys * kD * (E4m3 ? 1 : 2), kStage = 2 * kHalf, kStages = kRing / kStage;  // bytes of a warp's keys, or values
  static_assert(kStages <= kMaxStages, "barriers");
  extern __shared__ __align__(1024) unsigned char smem[];
  RowsShared &sh = *reinterpret_cast<RowsShared *>(smem + kWarps * kRing);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char *ring = smem + warp * kRing;
  const uint32_t ring_at = smem_u32(ring);
  const CacheIndex &ix = p.ix;

  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&sh.full[warp][i], 1);
    mbar_fence_init();
  }
  if (tid == 0) sh.abort = 0;
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  if (Redo && !__syncthreads_or(tid < p.looked && __ldcg(&p.any_redo[tid]) != 0)) return;

  // ------------------------------------------------------------------ the CTA's share
  auto tiles_of = [&](const Sequence &q) { return (int)(((long long)q.n * p.G + kRows - 1) / kRows); };
  auto span = [&](const Sequence &q, int t) {
    const int first = t * kRows, last = min((int)((long long)q.n * p.G), first + kRows) - 1;
    return span_of<kStep>(ix, q.len - q.n + first / p.G, q.len - q.n + last / p.G, q.len);
  };
  auto steps_of = [&](const Sequence &q, int &longest) -> long long {  // of one head
    long long n = 0;
    const int tiles = tiles_of(q);
    for (int t = 0; t < tiles; ++t) {
      const int k = span(q, t).steps;
      n += k;
      longest = max(longest, k);
    }
    return n;
  };
  auto quotient = [](long long a, long long b) -> long long {  // (of numbers that fit 32 bits as a rule: a tenth of the time)
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
  };
  Sequence q = {0, 0, 0};
  int s, longest = 1;
  long long share, u, u1, sequence_at, per_head;  // units of a CTA, its first one and the one behind its last; of the sequence, and of one of its heads
  bool one_tile = false;                          // shares do not cross tiles
  int h = 0, t = 0, done = 0;                     // head, tile and the tile's steps before this share
  // to be done again: the next tile of this CTA, whole
  long long pair = 0;
  auto next_redo = [&]() {
    const long long pairs = (long long)ix.S * p.Hkv;
    t += (int)gridDim.x;
    while (pair < pairs) {
      // the next one that is marked among 128, a lane four of them
      const long long base = pair & ~127LL, mine = base + lane * 4;
      uint32_t marks = 0u;
      if (mine + 3 >= pair && mine < pairs) {
        marks = __ldcg(reinterpret_cast<const uint32_t *>(p.redo + mine));
        if (mine < pair) marks &= 0xffffffffu << (8 * (int)(pair - mine));
        if (mine + 4 > pairs) marks &= 0xffffffffu >> (8 * (int)(mine + 4 - pairs));  // (bytes of no pair)
      }
      const uint32_t some = __ballot_sync(0xffffffffu, marks != 0u);
      if (some == 0u) {
        pair = base + 128;
        continue;
      }
      const int first = __ffs(some) - 1;
      pair = base + first * 4 + ((__ffs(__shfl_sync(0xffffffffu, marks, first)) - 1) >> 3);
      s = (int)(pair / p.Hkv);
      h = (int)(pair - (long long)s * p.Hkv);
      q = sequence(ix, s);
      const int tiles = tiles_of(q);
      if (t < tiles) return true;
      t -= tiles;
      ++pair;
    }
    return false;
  };
  if (Redo) {
    t = (int)blockIdx.x - (int)gridDim.x;
    if (!next_redo()) return;
    share = 1;
    sequence_at = per_head = u = 0;
    u1 = 1LL << 62;
  } else if (ix.S <= 32) {
    // every warp by itself, a lane a sequence
    if (lane < ix.S) q = sequence(ix, lane);
    per_head = steps_of(q, longest);
    longest = __reduce_max_sync(0xffffffffu, longest);
    auto before_lane = [&](long long x, long long &all) {
      const long long mine = x;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      all = __shfl_sync(0xffffffffu, x, 31);
      return x - mine;
    };
    long long total;
    sequence_at = before_lane(per_head * p.Hkv, total);
    share = max(quotient(total + gridDim.x - 1, gridDim.x), (long long)(longest + kMaxParts - 1) / kMaxParts);
    // Where each sequence and head is one tile and CTAs are enough, tiles begin with a share (a CTA with the end of one and the beginning of
    // another takes twice as long as the others: 8 heads x 4100 tokens).
    if (total < (1 << 20) && __all_sync(0xffffffffu, per_head == 0 || tiles_of(q) == 1)) {
      const int steps = (int)per_head;
      for (int more = 0; more <= (int)share / 4 + 1 && !one_tile; ++more) {
        const int sh1 = (int)share + more, parts = (steps + sh1 - 1) / sh1;
        if (__reduce_add_sync(0xffffffffu, parts * p.Hkv) <= (int)gridDim.x) {
          one_tile = true;
          share = sh1;
          per_head = (long long)parts * sh1;
        }
      }
      if (one_tile) sequence_at = before_lane(per_head * p.Hkv, total);
    }
    u = blockIdx.x * share;
    u1 = min(total, u + share);
    if (u >= u1) return;
    const uint32_t here = __ballot_sync(0xffffffffu, sequence_at <= u && u < sequence_at + per_head * p.Hkv);
    s = __ffs(here) - 1;
    q = {__shfl_sync(0xffffffffu, q.row, s), __shfl_sync(0xffffffffu, q.n, s), __shfl_sync(0xffffffffu, q.len, s)};
    sequence_at = __shfl_sync(0xffffffffu, sequence_at, s);
    per_head = __shfl_sync(0xffffffffu, per_head, s);
  } else {
    long long total = 0, mine = 0;
    for (int i = tid; i < ix.S; i += kThreads) {
      const Sequence x = sequence(ix, i);
      const long long n = steps_of(x, longest);
      if (i < kThreads) mine = n, q = x;
      total += n * p.Hkv;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, o);
      longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
    }
    if (lane == 0) {
      sh.total[warp] = total;
      sh.longest[warp] = longest;
    }
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      total += sh.total[i];
      longest = max(longest, sh.longest[i]);
    }
    share = max(quotient(total + gridDim.x - 1, gridDim.x), (long long)(longest + kMaxParts - 1) / kMaxParts);
    u = blockIdx.x * share;
    u1 = min(total, u + share);
    if (u >= u1) return;
    long long before = 0;  // steps before the sequences of this round
    for (int base = 0; base < ix.S; base += kThreads) {
      int dummy = 0;
      if (base > 0) {
        q = base + tid < ix.S ? sequence(ix, base + tid) : Sequence{0, 0, 0};
        mine = steps_of(q, dummy);
      }
      long long upto = mine * p.Hkv;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      __syncthreads();
      if (lane == 31) sh.total[warp] = upto;
      __syncthreads();
      long long at = before, all = 0;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) at += sh.total[i];
        all += sh.total[i];
      }
      at += upto - mine * p.Hkv;
      if (at <= u && u < at + mine * p.Hkv) {
        sh.found = base + tid;
        sh.found_q[0] = q.row, sh.found_q[1] = q.n, sh.found_q[2] = q.len;
        sh.found_at = at;
        sh.found_steps = mine;
      }
      before += all;
      if (before > u) break;
    }
    __syncthreads();
    s = sh.found;
    q = {sh.found_q[0], sh.found_q[1], sh.found_q[2]};
    sequence_at = sh.found_at;
    per_head = sh.found_steps;
  }
  if (!Redo) {
    long long rest = u - sequence_at;
    h = (int)quotient(rest, per_head);
    rest -= h * per_head;
    if (!one_tile)
      for (int k; rest >= (k = span(q, t).steps); ++t) rest -= k;
    done = (int)rest;
  }

  int put = 0, take = 0;            // the stages that come next, to fill and to use
  uint32_t parity = 0;              // of the barriers of the stages, a bit each, for their next use
  int in_flight = 0;
  bool ok = true;
  const int g = lane >> 2, c = lane & 3;
  const int box_log2 = min(ix.page_log2, kKeysLog2), boxes_log2 = kKeysLog2 - box_log2, boxes = 1 << boxes_log2;
  const int batch = 32 >> boxes_log2;  // steps whose entries of the table a warp asks for at once, a lane an entry

  // ---------------------------------------------------------------- a tile, or part of one
  int first_row, n_rows, p0, end_step, steps;
  int sinks, first;                                 // see Span
  int some_low, some_end, every_low, every_end;     // keys that some row sees, that every row does (besides the sinks)
  int next, next_batch, entry, entry_then;          // the warp's next copy; the batch of steps whose entries are in `entry`
  uint32_t qf[NT][8][2];
  auto some = [&](int k0) { return k0 < some_end && (k0 + kKeys > some_low || k0 < ix.sink); };
  auto key_of = [&](int i) { return (i < sinks ? i : first + i - sinks) * kStep + warp * kKeys; };
  auto entries = [&](int at) {  // of the steps from `at` on
    const int i = at + (lane >> boxes_log2), k = key_of(i) + ((lane & (boxes - 1)) << box_log2);
    return i < end_step && k < q.len ? page_entry(ix, s, k) : -1;
  };
  auto issue = [&]() {
    while (next < end_step && !some(key_of(next))) ++next;
    if (next >= end_step) return;
    while (next >= next_batch + batch) {
      next_batch += batch;
      entry = entry_then;
      entry_then = entries(next_batch + batch);
    }
    const int mine = __shfl_sync(0xffffffffu, entry, ((next - next_batch) << boxes_log2) + (lane & (boxes - 1)));
    uint64_t *bar = &sh.full[warp][put];
#ifdef HEART_TEST_HOOKS
    if (!(p.test_skip && blockIdx.x == 0 && warp == 0 && next == 1)) {
#endif
    if (lane == 0) mbar_expect_tx(bar, kStage + (E4m3 ? 2 * kKeys : 0));
    if (boxes > 1) __syncwarp();
    if (lane < boxes) {
      const int k0 = key_of(next), slot = k0 & ((1 << ix.page_log2) - 1);
      const int page = k0 + (lane << box_log2) < q.len ? checked_page(ix, mine) : ix.n_pages;  // (out of range: zeros)
      unsigned char *to = ring + put * kStage + (lane << (box_log2 + (E4m3 ? 7 : 8)));
      tma_load_5d(to, &map_k, bar, 0, slot, 0, h, page);
      tma_load_5d(to + kHalf, &map_v, bar, 0, slot, 0, h, page);
      if (E4m3) {
        const size_t at = (((size_t)page * p.Hkv + h) << ix.page_log2) + slot;
        bulk_load(&sh.scales[warp][put][lane << box_log2], page < ix.n_pages ? p.k_scale + at : kNoScales, 1 << box_log2, bar);
        bulk_load(&sh.scales[warp][put][kKeys + (lane << box_log2)], page < ix.n_pages ? p.v_scale + at : kNoScales, 1 << box_log2, bar);
      }
    }
#ifdef HEART_TEST_HOOKS
    }
#endif
    put = put + 1 == kStages ? 0 : put + 1;
    ++in_flight;
    ++next;
  };
  // What the tile needs before its first step, all that comes from memory asked for together; the first copies.
  auto start = [&]() {
    const Span<kStep> sp = span(q, t);
    sinks = sp.sinks, first = sp.first, steps = sp.steps;
    first_row = t * kRows;
    n_rows = min(kRows, (int)((long long)q.n * p.G) - first_row);
    p0 = q.len - q.n + first_row / p.G;
    const int p1 = q.len - q.n + (first_row + n_rows - 1) / p.G;
    end_step = (int)min((long long)steps, done + (u1 - u));
    next = done;
    next_batch = done;
    entry = entries(done);
    entry_then = entries(done + batch);
    const Visible a = visible(ix, max(p0, 0), q.len), b = visible(ix, p1, q.len);
    some_low = a.low, some_end = p1 < 0 ? 0 : b.end;
    every_low = b.low, every_end = p0 < 0 ? 0 : a.end;
    // The rows' queries as operands of the products, this lane's the row g of every 8.  (e4m3: the dims of a product are
    // those that a lane finds together in a key's row, 32 * c + 4 * step + 0 .. 3; as bf16 here, made f16 below.)
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const int row = m * 8 + g;
      const bool real = row < n_rows;
      const int i = (first_row + row) / p.G, head = h * p.G + (first_row + row) % p.G;
      const uint16_t *src = p.Q + (long long)(q.row + i) * p.qt + head * p.qh;
      if (E4m3) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4 x = real ? *reinterpret_cast<const uint4 *>(src + c * 32 + k * 8) : make_uint4(0u, 0u, 0u, 0u);
          qf[m][2 * k][0] = x.x;
          qf[m][2 * k][1] = x.y;
          qf[m][2 * k + 1][0] = x.z;
          qf[m][2 * k + 1][1] = x.w;
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          qf[m][ks][0] = real ? *reinterpret_cast<const uint32_t *>(src + ks * 16 + c * 2) : 0u;
          qf[m][ks][1] = real ? *reinterpret_cast<const uint32_t *>(src + ks * 16 + c * 2 + 8) : 0u;
        }
      }
    }
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) issue();
  };
  start();

  for (;;) {
    // Of the scores and sums a lane has the rows 2c and 2c + 1 of every 8.  (Rows that are none see everything, and nothing of theirs is kept.)
    Visible vis[NT][2];
    float row_scale[NT][2];
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      float scale = p.scale_log2;
      if (E4m3) {
        uint32_t top = 0u;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) top = __vmaxu2(top, __vmaxu2(qf[m][ks][0] & 0x7fff7fffu, qf[m][ks][1] & 0x7fff7fffu));
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max((int)(top >> 7) - 127 - 14, -100), 120);  // the largest element: 2^14 * 2^e to 2^15 * 2^e
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
        scale = top < 0x7f80u ? scale * __uint_as_float((uint32_t)(127 + e) << 23) : __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t w = qf[m][ks][k];
            qf[m][ks][k] = pack_f16x2(__uint_as_float(w << 16) * inv, __uint_as_float(w & 0xffff0000u) * inv);
          }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = m * 8 + c * 2 + r;
        row_scale[m][r] = E4m3 ? __shfl_sync(0xffffffffu, scale, (c * 2 + r) * 4) : scale;
        vis[m][r] = row < n_rows ? visible(ix, q.len - q.n + (first_row + row) / p.G, q.len) : Visible{0, 0x7fffffff};
      }
    }
    float o[NT][8][4] = {};
    float ref[NT][2], sum[NT][2];
    float sum_ref[NT][2];  // e4m3: of this lane's sums
#pragma unroll
    for (int m = 0; m < NT; ++m) ref[m][0] = ref[m][1] = sum_ref[m][0] = sum_ref[m][1] = kNoReference, sum[m][0] = sum[m][1] = 0.f;

#pragma unroll 1
    for (int i = done; i < end_step; ++i) {
      const int k0 = key_of(i);
      if (!some(k0)) continue;
      if (!mbar_wait(&sh.full[warp][take], (parity >> take) & 1, &sh.abort)) ok = false;
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const uint32_t k_at = ring_at + take * kStage, v_at = k_at + kHalf;
      const bool whole = k0 + kKeys <= every_end && (k0 >= every_low || k0 + kKeys <= ix.sink);
      float x[NT][kTiles][4] = {};
      float v_exp = 0.f;  // e4m3: the exponent of the value of key `lane`
      // ---- scores: keys g and g + 8 of every 16, rows 2c and 2c + 1
      if (E4m3) {
        // the scales, a lane a key: 2^e of the key (NaN where the token's key or value is not finite), e of the value
        const int key = lane & (kKeys - 1);
        const uint32_t kb = sh.scales[warp][take][key], vb = sh.scales[warp][take][kKeys + key];
        const float k_scale = cache_scale(vb == 255u ? 255u : kb);
        v_exp = (float)((int)vb - 127);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint4 lo = lds_u4(k_at + (t * 16 + g) * 128 + (((c * 2 + j) ^ g) << 4)), hi = lds_u4(k_at + (t * 16 + 8 + g) * 128 + (((c * 2 + j) ^ g) << 4));
            const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t a[4] = {codes_to_f16x2(l[k]), codes_to_f16x2(u[k]), high_codes_to_f16x2(l[k]), high_codes_to_f16x2(u[k])};
#pragma unroll
              for (int m = 0; m < NT; ++m) mma_f16(x[m][t], a, qf[m][j * 4 + k][0], qf[m][j * 4 + k][1]);
            }
          }
          const float f_lo = __shfl_sync(0xffffffffu, k_scale, t * 16 + g), f_hi = __shfl_sync(0xffffffffu, k_scale, t * 16 + 8 + g);
#pragma unroll
          for (int m = 0; m < NT; ++m) {
            x[m][t][0] *= f_lo;
            x[m][t][1] *= f_lo;
            x[m][t][2] *= f_hi;
            x[m][t][3] *= f_hi;
          }
        }
      } else {
        const int key = lane & 15;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const int chunk = ks * 2 + (lane >> 4);
          uint32_t a[4];
          ldmatrix4(a, k_at + (chunk >> 3) * 2048 + key * 128 + (((chunk ^ key) & 7) << 4));
#pragma unroll
          for (int m = 0; m < NT; ++m) mma_bf16(x[m][0], a, qf[m][ks][0], qf[m][ks][1]);
        }
      }
      // ---- weights
      auto hidden = [&](const Visible &v, int k) { return k >= v.end || (k < v.low && k >= ix.sink); };
      // Values that are not finite (codes that are no numbers) must not reach rows that do not see them (0 * inf is NaN): they are taken out, and
      // rows that do see them are marked.  (e4m3: ahead of the weights.  Behind them 64 single tokens over up to 16k took 255 us instead of 251.)
      auto look_at_values = [&]() {
        uint32_t bad = 0u;
        if (E4m3) {  // a lane a key, 16 bytes at a time in an order without bank conflicts
          uint32_t ends = 0u;  // a byte's top bit: 0x7f, 0xff
#pragma unroll 1
          for (int j = 0; j < 8; ++j) {
            const uint4 v = lds_u4(v_at + lane * 128 + ((j ^ (lane & 7)) << 4));
            ends |= ends_of(v.x) | ends_of(v.y) | ends_of(v.z) | ends_of(v.w);
          }
          bad = __ballot_sync(0xffffffffu, (ends & 0x80808080u) != 0u);
        } else {
#pragma unroll 1
          for (int j = 0; j < 8; ++j) {
            const uint4 v = lds_u4(v_at + (j * 32 + lane) * 16);
            if (not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w)) bad |= 1u << ((j * 4 + (lane >> 3)) & 15);
          }
          bad = __reduce_or_sync(0xffffffffu, bad);
        }
        if (bad) {
#pragma unroll 1
          for (int j = 0; j < 8; ++j)
            if (bad >> (E4m3 ? lane : (j * 4 + (lane >> 3)) & 15) & 1u)
              *reinterpret_cast<uint4 *>(ring + take * kStage + kHalf + (E4m3 ? lane * 128 + j * 16 : (j * 32 + lane) * 16)) = make_uint4(0u, 0u, 0u, 0u);
          async_proxy_fence();
          __syncwarp();
#pragma unroll 1
          for (uint32_t todo = bad; todo; todo &= todo - 1) {
            const int key = k0 + __ffs(todo) - 1;
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
              for (int r = 0; r < 2; ++r)
                if (!hidden(vis[m][r], key)) sum[m][r] = __uint_as_float(0x7fc00000u);
          }
        }
      };
      if (!whole) {
        if (E4m3) look_at_values();
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (hidden(vis[m][k & 1], k0 + t * 16 + g + (k >> 1) * 8)) x[m][t][k] = -INFINITY;
      }
      if (E4m3) {
        // the row sums, each lane's over its own keys; then scores with the exponents of the values
        auto sums = [&](auto masked) {
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              float top = -INFINITY;
#pragma unroll
              for (int t = 0; t < kTiles; ++t) top = fmaxf(top, fmaxf(x[m][t][r], x[m][t][2 + r]));
              top *= row_scale[m][r];
              if (top > sum_ref[m][r] + kMaxGrowth) {
                sum[m][r] *= ex2(sum_ref[m][r] - top);
                sum_ref[m][r] = top;
              }
            }
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const float e_lo = __shfl_sync(0xffffffffu, v_exp, t * 16 + g), e_hi = __shfl_sync(0xffffffffu, v_exp, t * 16 + 8 + g);
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float y = x[m][t][k], w = ex2(fmaf(y, row_scale[m][k & 1], -sum_ref[m][k & 1]));
                const float z = fmaf(y, row_scale[m][k & 1], k < 2 ? e_lo : e_hi);
                // (what is hidden is nothing, even to a query that is not finite)
                const bool none = decltype(masked)::value && y == -INFINITY;
                sum[m][k & 1] += none ? 0.f : w;
                x[m][t][k] = none ? -INFINITY : z;
              }
          }
        };
        if (whole) sums(False{});
        else sums(True{});
      }
      bool moved = false;
      float alpha[NT][2];
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float top = -INFINITY;
#pragma unroll
          for (int t = 0; t < kTiles; ++t) top = fmaxf(top, fmaxf(x[m][t][r], x[m][t][2 + r]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
          if (!E4m3) top *= row_scale[m][r];
          alpha[m][r] = 1.f;
          if (top > ref[m][r] + (E4m3 ? kHeadroomE4m3 : 0.f) + kMaxGrowth) {
            const float to = E4m3 ? top - kHeadroomE4m3 : top;
            alpha[m][r] = ex2(ref[m][r] - to);
            ref[m][r] = to;
            moved = true;
          }
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          if (!E4m3) {
            sum[m][0] *= alpha[m][0];
            sum[m][1] *= alpha[m][1];
          }
#pragma unroll
          for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[m][n][k] *= alpha[m][k & 1];
        }
      }
      uint32_t pf[NT][kTiles][2];  // as operands: row g, keys 2c, 2c + 1 of every 8
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          float w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = ex2(E4m3 ? x[m][t][k] - ref[m][k & 1] : fmaf(x[m][t][k], row_scale[m][k & 1], -ref[m][k & 1]));
          if (!E4m3) {
            sum[m][0] += w[0] + w[2];
            sum[m][1] += w[1] + w[3];
          }
          pf[m][t][0] = transposed(E4m3 ? pack_f16x2(w[0], w[1]) : pack_bf16x2(w[0], w[1]));
          pf[m][t][1] = transposed(E4m3 ? pack_f16x2(w[2], w[3]) : pack_bf16x2(w[2], w[3]));
        }
      if (!E4m3 && !whole) look_at_values();
      // ---- values: of every 16 dims the dims g and g + 8 (e4m3: 2g and 2g + 1), rows 2c and 2c + 1
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (E4m3) {
          const int key = lane & 15;
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            uint32_t b[4];
            const int chunk = j + (lane >> 4);
            ldmatrix4_trans(b, v_at + t * 2048 + key * 128 + (((chunk ^ key) & 7) << 4));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              // codes of two dims of a key and of the next: the even dims of both, the odd ones
              const uint32_t lo = __byte_perm(b[2 * k], 0, 0x3120), hi = __byte_perm(b[2 * k + 1], 0, 0x3120);
              const uint32_t a[4] = {codes_to_f16x2(lo), high_codes_to_f16x2(lo), codes_to_f16x2(hi), high_codes_to_f16x2(hi)};
#pragma unroll
              for (int m = 0; m < NT; ++m) mma_f16(o[m][j + k], a, pf[m][t][0], pf[m][t][1]);
            }
          }
        } else {
          const int key = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint32_t a[4];
            const int chunk = j * 2 + ((lane >> 3) & 1);
            ldmatrix4_trans(a, v_at + (chunk >> 3) * 2048 + key * 128 + (((chunk ^ key) & 7) << 4));
#pragma unroll
            for (int m = 0; m < NT; ++m) mma_bf16(o[m][j], a, pf[m][t][0], pf[m][t][1]);
          }
        }
      }
      __syncwarp();  // the stage has been read
      parity ^= 1u << take;
      take = take + 1 == kStages ? 0 : take + 1;
      --in_flight;
      issue();
    }
    if (!ok) {  // (copies that have not come are waited for once more, so that none lands in memory that is someone else's)
      for (; in_flight > 0; --in_flight) {
        const long long since = clock64();
        while (!mbar_try_wait(&sh.full[warp][take], (parity >> take) & 1) && clock64() - since < kWaitLimitCycles) {
        }
        parity ^= 1u << take;
        take = take + 1 == kStages ? 0 : take + 1;
      }
    }
    // ---------------------------------------------------------------- the warps' sums put together
    // A few rows have a place of their own, and the next tile's first copies go out ahead of this; more rows lie where the copies were.
    // (Pieces of 32 bytes are swizzled by the row.)
    const bool apart = n_rows <= kApartRows;
    unsigned char *sums = apart ? smem + kWarps * kRing + sizeof(RowsShared) : smem;
    const int sums_pitch = apart ? kApartRows * 512 : kRing;
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (E4m3) {
          float most = sum_ref[m][r];
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, k));
          sum[m][r] *= ex2(sum_ref[m][r] - most);
          sum_ref[m][r] = most;
        }
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) sum[m][r] += __shfl_xor_sync(0xffffffffu, sum[m][r], k);
        const int row = m * 8 + c * 2 + r;
        if (row >= n_rows) continue;
        if (g == 0) {
          sh.l[warp][row] = make_float2(sum[m][r], E4m3 ? sum_ref[m][r] : ref[m][r]);
          if (E4m3) sh.o_ref[warp][row] = ref[m][r];
        }
        unsigned char *to = sums + warp * sums_pitch + row * 512;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          if (E4m3) {
            *reinterpret_cast<float2 *>(to + ((n * 64 + g * 8) ^ ((row & 7) << 5))) = make_float2(o[m][n][r], o[m][n][2 + r]);
          } else {
            *reinterpret_cast<float *>(to + ((n * 64 + g * 4) ^ ((row & 7) << 5))) = o[m][n][r];
            *reinterpret_cast<float *>(to + ((n * 64 + 32 + g * 4) ^ ((row & 7) << 5))) = o[m][n][2 + r];
          }
        }
      }
    // this tile's, for the rest of it, before the next one's take their places
    const int rows = n_rows, row0 = first_row, out_row = q.row, out_head = h;
    const bool all = done == 0 && end_step == steps;
    const long long tile_at = u - done;  // the tile's first step
    const int tile_steps = steps;
    const int part = 2 * blockIdx.x + (done == 0 ? 1 : 0);
    u += end_step - done;
    const bool more = Redo ? next_redo() : !one_tile && u < u1;
    if (more) {
      done = 0;
      if (!Redo && ++t == tiles_of(q)) {
        t = 0;
        if (++h == p.Hkv) {
          h = 0;
          do q = sequence(ix, ++s);
          while (q.n == 0 && s + 1 < ix.S);
        }
      }
      if (apart) start();
    }
    __syncthreads();
    auto write_row = [&](int row, int d, float4 v, float l, float m) {  // four dims
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int i = (row0 + row) / p.G, head = out_head * p.G + (row0 + row) % p.G;
      *reinterpret_cast<uint2 *>(p.O + (long long)(out_row + i) * p.qt + head * p.qh + d) =
          make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
      if (d == 0 && p.lse != nullptr) p.lse[(long long)(out_row + i) * p.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    };
    const int d = lane * 4;
#pragma unroll 1
    for (int row = warp; row < rows; row += kWarps) {
      float m = kNoReference, m_o = kNoReference, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        m = fmaxf(m, sh.l[w][row].y);
        if (E4m3) m_o = fmaxf(m_o, sh.o_ref[w][row]);
      }
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 lm = sh.l[w][row];
        const float f = ex2(lm.y - m), f_o = E4m3 ? ex2(sh.o_ref[w][row] - m_o) : f;
        const float4 y = *reinterpret_cast<const float4 *>(sums + w * sums_pitch + row * 512 + ((d * 4) ^ ((row & 7) << 5)));
        l = fmaf(lm.x, f, l);
        v.x = fmaf(y.x, f_o, v.x);
        v.y = fmaf(y.y, f_o, v.y);
        v.z = fmaf(y.z, f_o, v.z);
        v.w = fmaf(y.w, f_o, v.w);
      }
      if (E4m3) {  // in units of the row sum
        const float f = ex2(m_o - m);
        v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
      }
      if (sh.abort) l = __uint_as_float(0x7fc00000u);
      if (all) {
        write_row(row, d, v, l, m);
      } else {
        __stcg(reinterpret_cast<float4 *>(p.parts + ((size_t)part * 128 + row) * 128 + d), v);
        if (lane == 0) __stcg(&p.part_l[part * 128 + row], make_float2(l, m));
      }
    }
    if (!all) {
      const int c0 = (int)quotient(tile_at, share), parts = (int)quotient(tile_at + tile_steps - 1, share) - c0 + 1;
      __syncthreads();
      if (tid == 0) {
        __threadfence();  // (of what the CTA has stored before the barrier)
        const bool last = atomicAdd(&p.arrivals[c0], 1) == parts - 1;
        if (last) p.arrivals[c0] = 0;
        sh.last = last;
        __threadfence();
      }
      __syncthreads();
      if (sh.last) {
#pragma unroll 1
        for (int row = warp; row < rows; row += kWarps) {
          auto place = [&](int i) { return (2 * (c0 + i) + (i == 0 ? 1 : 0)) * 128 + row; };
          const float2 mine = lane < parts ? __ldcg(&p.part_l[place(lane)]) : make_float2(0.f, kNoReference);  // (at most 32 parts)
          float m = mine.y;
#pragma unroll
          for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
          const float f = ex2(mine.y - m);
          float l = mine.x * f;
#pragma unroll
          for (int k = 16; k; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int i0 = 0; i0 < parts; i0 += 12) {
            float4 y[12];
#pragma unroll
            for (int k = 0; k < 12; ++k)
              if (i0 + k < parts) y[k] = __ldcg(reinterpret_cast<const float4 *>(p.parts + (size_t)place(i0 + k) * 128 + d));
#pragma unroll
            for (int k = 0; k < 12; ++k) {
              const float fk = __shfl_sync(0xffffffffu, f, (i0 + k) & 31);
              if (i0 + k < parts) {
                v.x = fmaf(y[k].x, fk, v.x);
                v.y = fmaf(y[k].y, fk, v.y);
                v.z = fmaf(y[k].z, fk, v.z);
                v.w = fmaf(y[k].w, fk, v.w);
              }
            }
          }
          write_row(row, d, v, l, m);
        }
      }
    }
    if (!more) break;
    if (!apart) async_proxy_fence();  // the rings held sums: behind them come copies
    __syncthreads();
    if (!apart) start();
  }
  if (tid == 0 && sh.abort) atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
}

}  // namespace

// A pool as (bytes of a row, slot, half row, head, page): a box is `rows` slots of one head, 128-byte rows, swizzled.
bool make_pool_map(CUtensorMap *m, const void *base, const CacheGeom &g, int rows, int halves) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const int bytes = g.e4m3 ? 1 : 2;
  cuuint64_t dims[5] = {(cuuint64_t)128 / bytes, (cuuint64_t)g.page, (cuuint64_t)bytes, (cuuint64_t)g.Hkv, (cuuint64_t)g.n_pages};
  cuuint64_t strides[4] = {(cuuint64_t)g.pt * bytes, 128, (cuuint64_t)g.ph * bytes, (cuuint64_t)g.pp * bytes};
  cuuint32_t box[5] = {(cuuint32_t)128 / bytes, (cuuint32_t)rows, (cuuint32_t)(g.e4m3 ? 1 : halves), 1, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(m, g.e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <int NT, bool E4m3, bool Redo>
cudaError_t launch(const CacheGeom &g, const RowsParams &p, const heart_cache &c, cudaStream_t s, int *launches) {
  const int box = g.page < keys_of(E4m3) ? g.page : keys_of(E4m3);
  CUtensorMap mk, mv;
  if (!make_pool_map(&mk, c.k, g, box, 2) || !make_pool_map(&mv, c.v, g, box, 2)) return cudaErrorInvalidValue;
  cudaError_t e = allow_shared_memory(cache_rows_kernel<NT, E4m3, Redo>, kRowsSmem);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_pdl(cache_rows_kernel<NT, E4m3, Redo>, dim3(kCacheCtas), dim3(kThreads), kRowsSmem, s, mk, mv, p);
}

RowsParams rows_params(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c, void *O, float *lse) {
  RowsParams p = {};
  p.ix = ix;
  p.Q = static_cast<const uint16_t *>(Q);
  p.O = static_cast<uint16_t *>(O);
  p.lse = lse;
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.qt = g.qt;
  p.qh = g.qh;
  p.Hq = g.Hq;
  p.Hkv = g.Hkv;
  p.G = g.G;
  p.scale_log2 = (float)(g.scale * 1.4426950408889634);
  p.test_skip = g.test_skip;
  p.arrivals = w.arrivals;
  p.parts = w.parts;
  p.part_l = w.part_l;
  return p;
}

}  // namespace

cudaError_t launch_cache_rows(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                              void *O, float *lse, cudaStream_t s, int *launches) {
  const RowsParams p = rows_params(g, ix, w, Q, c, O, lse);
  const bool eight = (long long)g.max_new * g.G <= 8;
  if (g.e4m3) return eight ? launch<1, true, false>(g, p, c, s, launches) : launch<2, true, false>(g, p, c, s, launches);
  return eight ? launch<1, false, false>(g, p, c, s, launches) : launch<2, false, false>(g, p, c, s, launches);
}

cudaError_t launch_cache_redo(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                              void *O, float *lse, int looked, cudaStream_t s, int *launches) {
  RowsParams p = rows_params(g, ix, w, Q, c, O, lse);
  p.test_skip = 0;
  p.redo = w.redo;
  p.any_redo = w.any_redo;
  p.looked = looked;
  return launch<2, true, true>(g, p, c, s, launches);
}

}  // namespace heart
