// Cross attention for many query rows a sequence and key head, on the sm_100a tensor cores.
//
// A tile is 128 rows: 128 / G tokens of a sequence with the G query heads of one key head.  Keys are processed 128 at a time, one CTA an SM, two
// softmax warpgroups that take the CTA's key steps in turn, scores double-buffered in tensor memory; the reasons are those at the top of attn_tc.cu, and so
// are what bounds it (the tensor pipe 1024 clocks a step, the special-function units 1024, shared memory 1280) and the way two warpgroups agree on a
// row's reference.  What differs, since all rows of a tile see the same keys and these are few (a text: 512, four steps):
//   * The end of a tile is the common case.  A warpgroup of its own takes the sums out of tensor memory, by way of registers, as bf16, into shared memory, from
//     where bulk copies write them, while the others are in the next tile's first steps.  Stores of all SMs go at some 10 bytes a clock and SM, 3000 clocks a tile:
//     a warpgroup that waited for its own would be late for the next tile's scores.  At each end every warp runs through other code than in between, and the
//     instruction cache does not hold all of it: little code a tile (loops that stay rolled, one wait in few instructions) gave more than fewer instructions.
//   * A tile's last step may have fewer than 128 keys: the products are cut to the next 16 keys (columns of the scores, 32 by pairs; steps of the values' product);
//     scores behind the last key become -inf in tensor memory, values of up to 15 rows behind it, which are anyone's, zeros in shared memory.
//   * Pairs of CTAs, for large calls, take two tiles of a sequence and head with half of the keys and of the values' dims each: the products of both are one
//     instruction of the first CTA's issuers, and half of the bytes come from L2.  Barriers that these wait for are the first CTA's, those that they complete both's.
//   * There is no plan: all tiles of a sequence take the same number of steps, so a CTA (or pair) finds its share of the line of all tiles' steps, (sequence, head,
//     tile, step), from the lengths alone, each beginning of a tile counted as kTileCost steps.
//     Parts of a tile go to the workspace; the CTA that brings the last one puts them together, in order: the result does not depend on which one
//     that is.
//
// Measured, 12 heads of 128, 20 calls after a pause: 32760 queries over 512 keys 108 us (955 TFLOP/s), over 128 54.7 (traffic: 202 MB, 3.7 TB/s), 4680 over 512 22.9, 1000 over 33k
// 182 (by pairs; 2 x 40 heads x 32760 over 343 518 us, 887 TFLOP/s and 2.6 TB/s).  Back to back for a second, at the power limit: 123, 58, 21, 212 and 600.
//
// Warp roles: 0-3, 4-7 softmax; 8 issues S = Q K^T; 9 copies V; 10 finds the CTA's parts, copies K and Q; 11 issues O += P V; 12-15 write.
// Tensor memory: O (128 columns) | S[2] (2 x 128) | P[2] (2 x 64).
// Every wait is bounded; one that runs out raises the CTA's abort flag and the status word, its roles stop, and what it owes to tiles that it shares
// is announced as no numbers, so that the workspace can be used again.
#include <algorithm>

#include "cross.cuh"
#include "tiles.cuh"

namespace heart {
using namespace tc;
namespace {

constexpr int kThreads = 512;
constexpr int kWarpQK = 8, kWarpV = 9, kWarpK = 10, kWarpPV = 11, kWarpOut = 12;
constexpr int kRegsSoftmax = 184, kRegsOut = 80, kRegsHelper = 64;  // 184 * 256 + 80 * 128 + 64 * 128 = the CTA's 512 x 128
static_assert(kRegsSoftmax * 256 + kRegsOut * 128 + kRegsHelper * 128 <= kThreads * 128, "registers at launch");
constexpr int kTileBytes = 32768;  // 128 rows x 128 dims: [2 dim halves][128 rows][64] bf16, 128-byte swizzle
constexpr int kTileCost = 1;       // of a tile besides its steps, in steps (as two the same; as three six prompts of 284 to 1256 over up to 474 states 35.8 us, not 32.2)
// Tiles of no more steps are not shared: an uneven finish costs half of a tile, parts 5 us.  (12 heads x 9000 over 1500, 12 steps, 78 us, 84 with parts; over 2000, 16
// steps, 100 and 105, but x 3500 53.6 and 52.5; over 2600, 21 steps, 127 and 133, but x 3500 66.9 and 63.)  Nor are tiles of no more than kPartsCost steps beside a CTA's share:
// where CTAs are left over, parts cost some ten steps.  (8 heads of 8 x 5 over 1250, 10 steps, 16.6 us, 16.3 with parts; over 2000, 16 steps, 21.2 and 17.6.)
constexpr long long kWholeSteps = 16, kPartsCost = 10;
constexpr int kPartRing = 4;
constexpr int kReaders = 15;       // of announced parts: softmax and writing warps, issuers, V producer
constexpr float kNoReference = -3.0e38f;
constexpr float kHeadroom = 16.f, kMaxGrowth = 8.f;  // see attn_tc.cu

// Part of a tile that a CTA takes: steps a .. b - 1.
struct alignas(16) Part {  // (written by fours)
  int row, tokens, h, key;  // first packed row, tokens, key head, first row of keys
  int4 steps;               // how many, keys of the last one, the tile's steps before them, 1 if they are all of the tile's; x < 0: no part left
  int c0, parts, pad[2];    // first CTA with a part of the tile, and how many there are
};

// Where a CTA is in the line of all tiles' costs.
struct Walk {
  Sequence q;
  int tiles, steps;      // of the sequence and a head, of a tile
  int s, h, tile, off;   // off: what of the tile's cost lies before the share
  long long u, end;      // of the line
};

// Sequences in a row: the length of their line, the largest cost of a tile.
struct alignas(16) Chunk {
  long long line;
  int longest;
};
static_assert(kThreads * sizeof(Chunk) <= kTileBytes, "they lie where rows are staged later");

template <bool Pair>
struct Ring {  // of keys and of values, of which a CTA of a pair has half
  static constexpr int kBytes = Pair ? kTileBytes / 2 : kTileBytes, kStages = 2 * kTileBytes / kBytes;
};
constexpr int kMostStages = 4;

struct CrossShared {
  uint64_t q_full[2], k_full[kMostStages], v_full[kMostStages];     // (those that an issuer waits for: of a pair, in its first CTA)
  uint64_t q_empty[2], k_empty[kMostStages], v_empty[kMostStages];  // the products have read it
  uint64_t l_ready[2][4], l_read[2];  // the row sum of the steps of the warpgroup without the last one is there, per lane quarter; the row sums have been read
  uint64_t l_final[2];     // the row sums are there for those who write (or in the workspace), per part & 1
  uint64_t v_tail;         // V_g is there, but for what is behind its last key
  uint64_t s_full[2], s_free[2], p_full[2], pv_done[2], m_ready[2][4];  // as in attn_tc.cu
  uint64_t o_full[2], o_free;
  uint64_t part_full[kPartRing], part_empty[kPartRing];
  uint64_t drain[2];
  uint64_t staged, stage_free;  // 64 dims of a tile's rows are in shared memory; have left it
  uint64_t finished;       // the other warps are through
  uint64_t stored;         // this CTA's part of a tile is in the workspace
  Part part[kPartRing];
  float m[128];            // references after the last step that has found them
  float l[2][128];         // of the row sums: the other warpgroup's part, then one over them, per part & 1
  uint32_t tmem_base;
  int shared_parts;        // parts of shared tiles that have been announced
  long long share;         // of the line, a CTA or a pair; 0: whole tiles
  int4 owed[2];            // this CTA's parts of shared tiles: place in the workspace, first CTA of the tile, number of its parts
  int n_owed;
  int4 merges[2];          // shared tiles that this CTA has brought the last part of: first row, tokens and key head, first CTA, number of parts
  int n_merges;
  int abort;
};
constexpr int kOffQ = 0, kOffK = 2 * kTileBytes, kOffV = 4 * kTileBytes, kOffStage = 6 * kTileBytes, kOffShared = kOffStage + kTileBytes;
constexpr int kSmem = kOffShared + sizeof(CrossShared);
static_assert(kSmem <= 232448, "shared memory of an SM");

struct CrossParams {
  CacheIndex ix;           // see launch_cross_rows
  int32_t *arrivals;
  float4 *parts;           // [2 * CTAs][32][128]: four dims of a row
  float2 *part_l;          // [2 * CTAs][128]
  uint16_t *O;
  float *lse;
  long long qt, qh;
  int Hq, Hkv, G;
  uint32_t inv_G;          // row / G = row * inv_G >> 16 for the rows of a tile
  float scale_log2;
  int test_skip;           // test-hook builds only: CTA 0 leaves out its second copy of values
};

__device__ __forceinline__ float reciprocal(float x) {  // (off by a unit in the last place at most)
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Waits for the barrier's phase of this parity; false if *abort is raised before.
__device__ __forceinline__ bool wait_unless(uint32_t bar, uint32_t parity, uint32_t abort) {
  uint32_t there;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b32 a;\n"
      "again:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 200000;\n\t"
      "@p bra done;\n\t"
      "ld.volatile.shared.u32 a, [%3];\n\t"
      "setp.eq.u32 p, a, 0;\n\t"
      "@p bra again;\n\t"
      "setp.ne.u32 p, a, a;\n"
      "done:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(there)
      : "r"(bar), "r"(parity), "r"(abort)
      : "memory");
  return there != 0;
}

template <bool Pair>
__global__ void __launch_bounds__(kThreads, 1)
    cross_tile_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const CrossParams p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  CrossShared &sh = *reinterpret_cast<CrossShared *>(smem + kOffShared);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const CacheIndex &ix = p.ix;
  volatile int *abort = &sh.abort;
  using R = Ring<Pair>;
  constexpr int kCtas = Pair ? 2 : 1;
  const int rank = Pair ? (int)cluster_ctarank() : 0, worker = blockIdx.x / kCtas, workers = gridDim.x / kCtas;
  // An arrival at, and a copy that counts on, a barrier of the CTA whose issuers wait for it.  (What an arrival says is ordered by the tensor memory's and the
  // copies' own fences.  As releases to the cluster two arrivals a step took 1000 clocks each.)
  auto arrive_first = [&](uint64_t *bar) {
    if (Pair) mbar_arrive_at(bar, 0);
    else mbar_arrive(bar);
  };
  auto expect = [&](uint64_t *bar, uint32_t bytes) {
    if (Pair) mbar_expect_tx_at(bar, 0, bytes);
    else mbar_expect_tx(bar, bytes);
  };
  auto copy = [&](void *dst, const CUtensorMap *map, uint64_t *bar, int c1, int c2, int c3, int c4) {
    if (Pair) tma_load_5d_pair(dst, map, cluster_address(smem_u32(bar), 0), 0, c1, c2, c3, c4);
    else tma_load_5d(dst, map, bar, 0, c1, c2, c3, c4);
  };
  auto commit = [&](uint64_t *bar) {  // in both CTAs
    if (Pair) tc_commit_pair(bar);
    else tc_commit(bar);
  };

  // ------------------------------------------------------------------ set-up
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], kCtas);
      mbar_init(&sh.q_empty[i], 1);
      mbar_init(&sh.l_read[i], 4);
      mbar_init(&sh.l_final[i], 4);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], 4 * kCtas);
      mbar_init(&sh.p_full[i], 4 * kCtas);
      mbar_init(&sh.pv_done[i], 1);
      for (int q = 0; q < 4; ++q) {
        mbar_init(&sh.m_ready[i][q], 1);
        mbar_init(&sh.l_ready[i][q], 1);
      }
      mbar_init(&sh.o_full[i], 1);
      mbar_init(&sh.drain[i], 1);
    }
    for (int i = 0; i < R::kStages; ++i) {
      mbar_init(&sh.k_full[i], kCtas);
      mbar_init(&sh.v_full[i], kCtas);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_empty[i], 1);
    }
    for (int i = 0; i < kPartRing; ++i) {
      mbar_init(&sh.part_full[i], 1);
      mbar_init(&sh.part_empty[i], rank == 0 ? kReaders : kReaders - 2);  // (the second CTA has no issuers)
    }
    mbar_init(&sh.v_tail, 1);
    mbar_init(&sh.o_free, 4 * kCtas);
    mbar_init(&sh.staged, 4);
    mbar_init(&sh.stage_free, 1);
    mbar_init(&sh.stored, 4);
    mbar_init(&sh.finished, kThreads / 32 - 1);
    sh.abort = 0;
    sh.shared_parts = sh.n_owed = sh.n_merges = 0;
    mbar_fence_init();
  }
  if (warp == kWarpK && lane == 0) {
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    tma_prefetch_desc(&map_o);
  }
  if (warp == kWarpQK) {
    if (Pair) {
      tmem_alloc_pair(&sh.tmem_base, 512);
    } else {
      tmem_alloc(&sh.tmem_base, 512);
      tmem_relinquish();
    }
  }
  pdl_wait();
  pdl_launch_dependents();

  // ------------------------------------------------------------------ the CTA's share of the line
  const int tokens_per_tile = 128 / p.G;
  auto tiles_of = [&](const Sequence &q) {  // or pairs of them
    return (int)(((long long)q.n + kCtas * tokens_per_tile - 1) / (kCtas * tokens_per_tile));
  };
  auto steps_of = [&](const Sequence &q) { return max((q.len + kKeyStep - 1) / kKeyStep, 1); };  // (one without any key: the rows are written)
  auto cost_of = [&](const Sequence &q) { return steps_of(q) + kTileCost; };
  auto quotient = [](long long a, long long b) -> long long {  // (little code: of numbers that fit 32 bits as a rule, of others a bit at a time)
    if (((a | b) >> 32) == 0) return (long long)((uint32_t)a / (uint32_t)b);
    long long q = 0, r = 0;
#pragma unroll 1
    for (int i = 62; i >= 0; --i) {
      r = r << 1 | (a >> i & 1);
      q <<= 1;
      if (r >= b) r -= b, q |= 1;
    }
    return q;
  };
  auto line_of = [&](const Sequence &q) { return (long long)tiles_of(q) * cost_of(q) * p.Hkv; };
  SequenceWords of_lane = {0, 0, 0, 0};
  // More than 32 sequences: what they cost, some in a row a thread, for the K producer.
  Chunk *const chunks = reinterpret_cast<Chunk *>(smem + kOffStage);
  const int per_chunk = (ix.S + kThreads - 1) / kThreads, n_chunks = (ix.S + per_chunk - 1) / per_chunk;
  if (ix.S > 32) {
    if (tid < n_chunks) {
      Chunk mine = {0, 1};
#pragma unroll 1
      for (int i = tid * per_chunk; i < min(ix.S, (tid + 1) * per_chunk); ++i) {
        const Sequence q = cross_sequence(ix, i);
        const long long line = line_of(q);
        mine.line += line;
        if (line > 0) mine.longest = max(mine.longest, cost_of(q));
      }
      chunks[tid] = mine;
    }
  } else if (warp == kWarpK && lane < ix.S) {  // a lane a sequence
    of_lane = cross_sequence_words(ix, lane);  // (they are looked at behind the barrier)
  }
  tc_fence_before();
  if (Pair) cluster_sync();  // (the other CTA's barriers are there)
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;

  // Waits of a whole warp; ok turns false when the CTA aborts.  Little code: it stands in many places.  What bounds them all is the K producer's clock: nothing goes
  // on for long when one of its copies' places does not become free, and at the end it waits for the other warps.
  bool ok = true;
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    return ok = __all_sync(0xffffffffu, wait_unless(smem_u32(bar), parity, smem_u32(&sh.abort)));
  };
  auto timed_wait = [&](uint64_t *bar, uint32_t parity) {
    const uint32_t since = clock();
#pragma unroll 1
    while (__builtin_expect(!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)), 0)) {
      if (__any_sync(0xffffffffu, *abort != 0 || (uint32_t)clock() - since > (uint32_t)kWaitLimitCycles)) {
        *abort = 1;
        if (Pair) cluster_st1(cluster_address(smem_u32(&sh.abort), rank ^ 1), 1u);
        return ok = false;
      }
    }
    return ok;
  };
  auto wait2 = [&](uint64_t *bar0, uint32_t parity0, uint64_t *bar1, uint32_t parity1) {  // (one after the other, by the same instructions)
#pragma unroll 1
    for (int i = 0; i < 2; ++i)
      if (!wait(i == 0 ? bar0 : bar1, i == 0 ? parity0 : parity1)) break;
    return ok;
  };
  // The announced part n; nullptr: abort.
  auto part_at = [&](int n) -> const Part * {
    if (!wait(&sh.part_full[n % kPartRing], (n / kPartRing) & 1)) return nullptr;
    return &sh.part[n % kPartRing];
  };
  auto done_with_part = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_empty[n % kPartRing]);
  };
  // Of up to 128 keys, those that the products take: of values 16 at a time, of scores 16 or, by pairs, 32.
  auto values_read = [](int keys) { return min(max((keys + 15) & ~15, 16), kKeyStep); };
  auto keys_read = [](int keys) { return min(max((keys + 16 * kCtas - 1) & ~(16 * kCtas - 1), 16 * kCtas), kKeyStep); };
  auto settle = [&](uint64_t *bar, uint32_t parity) {
    const uint32_t t0 = clock();
    while (!mbar_try_wait(bar, parity) && (uint32_t)clock() - t0 < 40000000u) {
    }
  };
  auto desc_at = [](uint64_t desc, uint32_t off16) -> uint64_t {
    return (desc & 0xffffffff00000000ull) | (uint32_t)((uint32_t)desc + off16);
  };
  auto drain_products = [&](bool leader, uint64_t *bar) {
    if (!*abort) return;
    if (leader) commit(bar);
    __syncwarp();
    settle(bar, 0);
  };
  auto lse_of = [&](int first, int h, int row) {
    const int t = (int)(((uint32_t)row * p.inv_G) >> 16);
    return p.lse + (long long)(first + t) * p.Hq + h * p.G + row - t * p.G;
  };

  // ------------------------------------------------------------------ roles
  // (Each warpgroup's registers are set where its code begins: behind a place where two come together again the compiler counts on the smaller number.)
  if (warp >= kWarpOut) {
    // ===== output: thread = one row
    setmaxnreg_dec<kRegsOut>();
    const uint32_t quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t o_addr = tmem + (quarter << 21);
    const uint32_t stage_at = smem_u32(smem + kOffStage) + row * 128;
    uint32_t n_stored = 0, n_staged = 0;
    auto load = [&](uint32_t (&v)[32], int quad) {
      tmem_ld32(o_addr + quad * 32, v);
      tmem_wait_ld();
    };
    auto loaded = [&]() {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_first(&sh.o_free);
    };
    // 32 dims of the row as bf16, O / l, and into shared memory
    auto pack = [&](const uint32_t (&v)[32], float inv, uint32_t (&y)[16]) {
      const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float a0, a1;
        unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), inv2), a0, a1);
        y[i] = pack_bf16x2(a0, a1);
      }
    };
    auto stage = [&](const uint32_t (&y)[16], int quad) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sts_u4(stage_at + (quad >> 1) * (kTileBytes / 2) + ((((quad & 1) * 4 + i ^ lane) & 7) << 4), make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]));
    };
    auto stage_free = [&]() {  // once the tile before has left
      if (n_staged == 0) return true;
      if (quarter == 0 && lane == 0) {
        bulk_wait_read();
        mbar_arrive(&sh.stage_free);
      }
      __syncwarp();
      return wait(&sh.stage_free, (n_staged - 1) & 1);
    };
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr || x->steps.x < 0) break;
      const bool all = x->steps.w != 0;
      // (The row sums are ordinary stores of this CTA's threads.  By pairs o_full comes by way of the first CTA's issuers, which orders tensor memory only.  A barrier more a tile: no difference.)
      if (!wait2(&sh.o_full[n & 1], (n >> 1) & 1, &sh.l_final[n & 1], (n >> 1) & 1)) break;
      tc_fence_after();
      if (__builtin_expect(all, 1)) {
        const float inv = sh.l[n & 1][row];
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.l_read[n & 1]);
        if (!stage_free()) break;
#pragma unroll
        for (int quad = 0; quad < 4; ++quad) {
          uint32_t v[32], y[16];
          load(v, quad);
          if (quad == 3) loaded();
          pack(v, inv, y);
          stage(y, quad);
        }
      } else {
        // part of a shared tile: its sums to the workspace (the row sums are there); whoever brings the last one puts them together when all else is done
        if (lane == 0) mbar_arrive(&sh.l_read[n & 1]);
        const bool real = row < x->tokens * p.G;
        const int slot = 2 * blockIdx.x + (x->steps.z == 0 ? 1 : 0);
#pragma unroll 1
        for (int d = 0; d < 128; d += 32) {
          uint32_t v[32];
          load(v, d >> 5);
          if (d == 96) loaded();
          float4 *const to = &p.parts[(size_t)(slot * 32 + (d >> 2)) * 128 + row];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (real)
              __stcg(to + k * 128, make_float4(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]), __uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3])));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.stored);
        if (quarter == 0) {
          if (!wait(&sh.stored, n_stored & 1)) break;
          if (lane == 0) {
            __threadfence();  // (of what the CTA has stored, which the barriers have shown this thread)
            int32_t *const arrivals = &p.arrivals[x->c0 * kCtas + rank];
            if (atomicAdd(arrivals, 1) == x->parts - 1) {
              *arrivals = 0;
              sh.merges[sh.n_merges++] = make_int4(x->row, x->tokens | x->h << 8, x->c0, x->parts);
            }
            ++sh.shared_parts;
            __threadfence();
          }
          __syncwarp();
        }
        ++n_stored;
        done_with_part(n);
        continue;
      }
      async_proxy_fence();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.staged);
      const bool whole_tile = x->tokens == tokens_per_tile;
      if (quarter == 0) {
        if (!wait(&sh.staged, n_staged & 1)) break;
        if (lane == 0 && whole_tile) {
          tma_store_5d(&map_o, smem + kOffStage, 0, 0, x->row, 0, x->h);
          tma_store_5d(&map_o, smem + kOffStage + kTileBytes / 2, 0, 0, x->row, 1, x->h);
        }
        __syncwarp();
      }
      ++n_staged;
      if (__builtin_expect(!whole_tile, 0)) {  // the rows that there are, two at a time, 16 lanes each
        uint16_t *const to = p.O + (long long)x->row * p.qt + (long long)(x->h * p.G) * p.qh + (lane & 15) * 8;
        const uint32_t from = smem_u32(smem + kOffStage) + ((lane & 15) >> 3) * (kTileBytes / 2);
#pragma unroll 1
        for (int r = (int)quarter * 32 + (lane >> 4); r < min(x->tokens * p.G, (int)quarter * 32 + 32); r += 2) {
          const int t = (int)(((uint32_t)r * p.inv_G) >> 16);
          *reinterpret_cast<uint4 *>(to + (long long)t * p.qt + (long long)(r - t * p.G) * p.qh) = lds_u4(from + r * 128 + (((lane ^ r) & 7) << 4));
        }
      }
      done_with_part(n);
    }
    if (quarter == 0 && lane == 0) bulk_wait_read();
  } else if (warp >= kWarpQK) {
    setmaxnreg_dec<kRegsHelper>();
    if (warp == kWarpK) {
      // ===== the CTA's parts; K and Q producer
      Walk w = {};
      auto next_sequence = [&]() {
        w.q = cross_sequence(ix, ++w.s);
        w.tiles = tiles_of(w.q);
        w.steps = steps_of(w.q);
      };
      {
        const bool few = ix.S <= 32;
        const Sequence sequence = few && lane < ix.S ? cross_sequence(ix, of_lane) : Sequence{0, 0, 0, 0};
        const int lanes = few ? ix.S : 32;  // that there are sequences or chunks for
        auto upto_lane = [&](long long x) {  // inclusive, over those
#pragma unroll 1
          for (int o = 1; o < lanes; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
          }
          return x;
        };
        long long total = line_of(sequence);
        int longest = total > 0 ? cost_of(sequence) : 1;
#pragma unroll 1
        for (int i = few ? n_chunks : lane; i < n_chunks; i += 32) {
          total += chunks[i].line;
          longest = max(longest, chunks[i].longest);
        }
        long long mine = total, upto = upto_lane(mine);
        total = __shfl_sync(0xffffffffu, upto, lanes - 1);
        longest = __reduce_max_sync(0xffffffffu, longest);
        // (A part takes the CTA that puts a tile together 0.6 us, 64 KB at 55 bytes a clock, a step 0.8: of few long tiles about as many parts as steps a part.  4 heads x 300
        // over 4000 23.0 us, with 11 parts a tile 24.8; x 128 over 9000 25.6, with 16 29.9.)
        const long long even = quotient(total + workers - 1, workers), least = (long long)sqrtf((float)longest);
        const bool whole = longest <= min(kWholeSteps + kTileCost, max(even, least) + kPartsCost);  // tiles are not shared: a CTA takes those that begin in its share
        const long long share = whole ? max(even, 1LL) : max(even, least);
        if (lane == 0) sh.share = whole ? 0 : share;
        w.u = worker * share;
        w.end = min(total, w.u + share);
        if (w.u < w.end) {  // the chunk in which the share begins, then the sequence (all lanes alike)
          long long before = 0;
          int chunk = 0;
#pragma unroll 1
          for (;; chunk += 32) {
            if (!few) {
              mine = chunk + lane < n_chunks ? chunks[chunk + lane].line : 0;
              upto = before + upto_lane(mine);
            }
            const uint32_t here = __ballot_sync(0xffffffffu, lane < lanes && w.u < upto);
            const int at = here ? __ffs(here) - 1 : 31;
            before = __shfl_sync(0xffffffffu, here ? upto - mine : upto, at);
            if (here) {
              chunk += at;
              break;
            }
          }
          if (few) {
            w.s = chunk;
            w.q = {__shfl_sync(0xffffffffu, sequence.row, chunk), __shfl_sync(0xffffffffu, sequence.n, chunk), __shfl_sync(0xffffffffu, sequence.len, chunk),
                   __shfl_sync(0xffffffffu, sequence.key, chunk)};
            w.tiles = tiles_of(w.q);
            w.steps = steps_of(w.q);
          } else {
            w.s = chunk * per_chunk - 1;
#pragma unroll 1
            for (long long line = 0;; before += line) {
              next_sequence();
              line = (long long)w.tiles * (w.steps + kTileCost) * p.Hkv;
              if (w.u < before + line) break;
            }
          }
          const long long rest = w.u - before, at = quotient(rest, w.steps + kTileCost);  // tile of all heads
          w.off = (int)(rest - at * (w.steps + kTileCost));
          w.h = (int)quotient(at, w.tiles);
          w.tile = (int)(at - (long long)w.h * w.tiles);
          if (whole && w.off > 0) {
            w.u += w.steps + kTileCost - w.off;
            ++w.tile;
            w.off = 0;
          }
        }
        __syncwarp();
      }
      // Part n + 1 is announced with the first step of part n.
      // (Little code for a tile like the one before, in registers: K waits for it.  By one thread from shared memory it took 2400 clocks, and 12 heads x 32760 over 512
      // 112 us.)  n = -1: no steps.
      int g = 0, n_steps = 1, ends = 0, h = 0, key = 0, row = 0;
      bool any = true;
#pragma unroll 1
      for (int n = -1; any; ++n) {
#pragma unroll 1
        for (int i = 0; i < n_steps; ++i) {
          const int st = g % R::kStages;
          if (n >= 0 && ok && (g < R::kStages || timed_wait(&sh.k_empty[st], (g / R::kStages - 1) & 1))) {
            if (lane == 0) {  // (of a pair's products each CTA has half of the keys that they take)
              expect(&sh.k_full[st], R::kBytes);
              copy(smem + kOffK + st * R::kBytes, &map_k, &sh.k_full[st], key + rank * (keys_read(i == n_steps - 1 ? ends : kKeyStep) >> 1), 0, h, 0);
            }
            ++g;
            key += kKeyStep;
            if (i == 0 && (n < 2 || timed_wait(&sh.q_empty[n & 1], ((n - 2) >> 1) & 1)) && lane == 0) {
              unsigned char *q = smem + kOffQ + (n & 1) * kTileBytes;
              expect(&sh.q_full[n & 1], 2 * (128 / p.G * p.G) * 128);
              copy(q, &map_q, &sh.q_full[n & 1], 0, row, 0, h);
              copy(q + kTileBytes / 2, &map_q, &sh.q_full[n & 1], 0, row, 1, h);
            }
            __syncwarp();
          }
          if (i == 0) {
            const int m = n + 1;
            if (ok && m >= kPartRing) timed_wait(&sh.part_empty[m % kPartRing], (m / kPartRing - 1) & 1);
            Part &x = sh.part[m % kPartRing];  // (this warp alone writes the ring)
            // the tile at u
            any = w.u < w.end;
            if (any) {
              if (__builtin_expect(w.tile == w.tiles, 0)) {
                w.tile = 0;
                if (++w.h == p.Hkv) {
                  w.h = 0;
#pragma unroll 1
                  do next_sequence();
                  while (w.tiles == 0 && w.s + 1 < ix.S);
                }
              }
              int a = 0, b = w.steps, c0 = worker, parts = 1;
              const long long tile_at = w.u - w.off;
              if (__builtin_expect(w.off > 0 || w.end - w.u < w.steps + kTileCost, 0)) {
                const long long share = sh.share;
                if (share > 0) {
                  a = max(w.off - kTileCost, 0);
                  b = (int)min((long long)w.steps, w.end - tile_at - kTileCost);
                  if (b - a < w.steps) {
                    c0 = (int)quotient(tile_at + kTileCost, share);
                    parts = (int)quotient(tile_at + kTileCost + w.steps - 1, share) - c0 + 1;
                  }
                  any = b > a;  // (else the share ends before the tile's first step)
                }
              }
              if (any) {
                const int first = (w.tile * kCtas + rank) * tokens_per_tile;
                if (lane == 0) {
                  if (parts > 1) sh.owed[sh.n_owed++] = make_int4(2 * blockIdx.x + (a == 0 ? 1 : 0), c0 * kCtas + rank, parts, 0);
                  if (ok) {  // (after an abort only what is owed is put down)
                    int4 *const to = reinterpret_cast<int4 *>(&x);
                    to[0] = make_int4(w.q.row + first, min(tokens_per_tile, max(w.q.n - first, 0)), w.h, w.q.key + a * kKeyStep);
                    to[1] = make_int4(b - a, b < w.steps ? kKeyStep : w.q.len - (w.steps - 1) * kKeyStep, a, b - a == w.steps);
                    to[2] = make_int4(c0, parts, 0, 0);
                  }
                }
                w.u = tile_at + kTileCost + b;
                w.off = 0;
                ++w.tile;
              }
            }
            if (lane == 0 && ok) {
              if (!any) x.steps.x = -1;
              mbar_arrive(&sh.part_full[m % kPartRing]);
            }
            __syncwarp();
          }
          if (!ok) break;
        }
        const Part &x = sh.part[(n + 1) % kPartRing];
        const int4 head = *reinterpret_cast<const int4 *>(&x);
        n_steps = x.steps.x, ends = x.steps.y, row = head.x, h = head.z, key = head.w;
        if (!ok) n_steps = 1;
      }
      if (ok) timed_wait(&sh.finished, 0);
    } else if (warp == kWarpV) {
      // ===== V producer
      int g = 0;
      uint32_t tails = 0;
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        const Part *x = part_at(n);
        if (x == nullptr || x->steps.x < 0) break;
        const int4 steps = x->steps;
        const int n_steps = steps.x, h = x->h, key = x->key;
        done_with_part(n);
#pragma unroll 1
        for (int i = 0; i < n_steps; ++i, ++g) {
          const int st = g % R::kStages;
          if (g >= R::kStages && !wait(&sh.v_empty[st], (g / R::kStages - 1) & 1)) break;
          unsigned char *const to = smem + kOffV + st * R::kBytes;
          const int keys = i == n_steps - 1 ? steps.y : kKeyStep;
          const bool tail = (keys & 15) || keys == 0;
#ifdef HEART_TEST_HOOKS
          if (!(p.test_skip && blockIdx.x == 0 && g == 1))
#endif
          if (lane == 0) {  // (of a pair's products each CTA has half of the dims)
            if (tail) {
              mbar_expect_tx(&sh.v_tail, R::kBytes);
              tma_load_5d(to, &map_v, &sh.v_tail, 0, key + i * kKeyStep, rank, h, 0);
            } else {
              expect(&sh.v_full[st], R::kBytes);
              copy(to, &map_v, &sh.v_full[st], key + i * kKeyStep, rank, h, 0);
            }
          }
          __syncwarp();
          if (tail) {  // rows that a product reads behind the last key
            if (!wait(&sh.v_tail, tails & 1)) break;
            ++tails;
            const int out = keys == 0 ? 16 : 16 - (keys & 15);
#pragma unroll 1
            for (int j = lane; j < out * 8 * (2 / kCtas); j += 32) {
              const int half = Pair ? 0 : j & 1, at = Pair ? j : j >> 1;
              sts_u4(smem_u32(to) + half * (kTileBytes / 2) + (keys + (at >> 3)) * 128 + (at & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
            }
            async_proxy_fence();
            __syncwarp();
            if (lane == 0) {
              if (Pair) mbar_arrive_in(&sh.v_full[st], 0);
              else mbar_arrive(&sh.v_full[st]);
            }
          }
        }
      }
    } else if (rank != 0) {
      // (the issuers of a pair are the first CTA's)
    } else if (warp == kWarpQK) {
      // ===== issuer of the score products
      const uint64_t q_desc = smem_desc_sw128(smem_u32(smem + kOffQ), 16, 1024);
      const uint64_t k_desc = smem_desc_sw128(smem_u32(smem + kOffK), 16, 1024);
      const bool leader = elect_one();
      uint32_t g = 0;
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        const Part *x = part_at(n);
        if (x == nullptr || x->steps.x < 0) break;
        const int n_steps = x->steps.x, ends = x->steps.y;
        done_with_part(n);
        wait(&sh.q_full[n & 1], (n >> 1) & 1);
        const uint64_t qd = desc_at(q_desc, (n & 1) * (kTileBytes >> 4));
#pragma unroll 1
        for (int i = 0; i < n_steps; ++i, ++g) {  // S_g = Q K_g^T
          const uint32_t b = g & 1;
          const uint32_t st = g % R::kStages;
          if (!wait2(&sh.s_free[b], ((g - 2) >> 1) & 1, &sh.k_full[st], (g / R::kStages) & 1)) break;  // (the phase before the first one counts as past)
          tc_fence_after();
          if (leader) {
            const uint64_t kd = desc_at(k_desc, st * (R::kBytes >> 4));
            const int keys = i == n_steps - 1 ? keys_read(ends) : kKeyStep;
            const uint32_t idesc = idesc_bf16_f32(128 * kCtas, 0, false, false) | (uint32_t)(keys >> 3) << 17;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
              const uint64_t qk = desc_at(qd, (ks >> 2) * 1024 + (ks & 3) * 2), kk = desc_at(kd, (ks >> 2) * (R::kBytes >> 5) + (ks & 3) * 2);
              if (Pair) mma_ss_pair(tmem + 128 + b * 128, qk, kk, idesc, ks > 0 ? 1u : 0u);
              else mma_ss(tmem + 128 + b * 128, qk, kk, idesc, ks > 0 ? 1u : 0u);
            }
            commit(&sh.s_full[b]);
            commit(&sh.k_empty[st]);
            if (i == n_steps - 1) commit(&sh.q_empty[n & 1]);
          }
          __syncwarp();
        }
      }
      drain_products(leader, &sh.drain[0]);
    } else if (warp == kWarpPV) {
      // ===== issuer of the value products
      constexpr uint32_t idesc = idesc_bf16_f32(128 * kCtas, 128, false, true);
      const uint64_t v_desc = smem_desc_sw128(smem_u32(smem + kOffV), kTileBytes / 2, 1024);
      const bool leader = elect_one();
      uint32_t g = 0;
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        const Part *x = part_at(n);
        if (x == nullptr || x->steps.x < 0) break;
        const int n_steps = x->steps.x, ends = x->steps.y;
        done_with_part(n);
        if (n > 0) wait(&sh.o_free, (n - 1) & 1);
#pragma unroll 1
        for (int i = 0; i < n_steps; ++i, ++g) {  // O (+)= P_g V_g
          const uint32_t b = g & 1;
          const uint32_t st = g % R::kStages;
          if (!wait2(&sh.v_full[st], (g / R::kStages) & 1, &sh.p_full[b], (g >> 1) & 1)) break;
          // (the other CTA's zeros behind the last key are ordinary stores.  By a fence 2 x 12 heads x 32760 over 343 took 209 us, not 184, the same as without any.)
          if (Pair && i == n_steps - 1 && ((ends & 15) || ends == 0)) mbar_acquire_cluster(&sh.v_full[st], (g / R::kStages) & 1);
          tc_fence_after();
          if (leader) {
            const uint64_t vd = desc_at(v_desc, st * (R::kBytes >> 4));
            const int ks_end = i == n_steps - 1 ? values_read(ends) >> 4 : 8;
            auto product = [&](int ks) {
              const uint64_t at = desc_at(vd, ks * 128);
              if (Pair) mma_ts_pair(tmem, tmem + 384 + b * 64 + ks * 8, at, idesc, (i > 0 || ks > 0) ? 1u : 0u);
              else mma_ts(tmem, tmem + 384 + b * 64 + ks * 8, at, idesc, (i > 0 || ks > 0) ? 1u : 0u);
            };
            if (__builtin_expect(ks_end == 8, 1)) {
#pragma unroll
              for (int ks = 0; ks < 8; ++ks) product(ks);
            } else {
#pragma unroll 1
              for (int ks = 0; ks < ks_end; ++ks) product(ks);
            }
            if (i == n_steps - 1) commit(&sh.o_full[n & 1]);
            commit(&sh.pv_done[b]);
            commit(&sh.v_empty[st]);
          }
          __syncwarp();
        }
      }
      drain_products(leader, &sh.drain[1]);
    }
  } else {
    // ===== softmax: thread = one row; warpgroup w takes the steps g with g & 1 == w
    setmaxnreg_inc<kRegsSoftmax>();
    const uint32_t w = warp >> 2, quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t o_addr = tmem + (quarter << 21), s_at = o_addr + 128 + w * 128, p_at = o_addr + 384 + w * 64;
    const float c = p.scale_log2;
    const uint64_t c2 = pack_f32x2(c, c);
    auto arrive = [&](uint64_t *bar) {  // this warp's tensor-memory accesses so far are ordered before it
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_first(bar);
    };
    uint32_t g0 = 0;  // key steps before the present part
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int4 steps = x->steps;
      const int n_steps = steps.x, ends = steps.y;
      if (n_steps < 0) break;
      float m_ref = kNoReference, l_run = 0.f;
#pragma unroll 1
      for (int h = (w ^ g0) & 1; h < n_steps; h += 2) {
        const uint32_t g = g0 + h;
        if (!wait(&sh.m_ready[w ^ 1][quarter], ((g - 1) >> 1) & 1) || !wait(&sh.s_full[w], (g >> 1) & 1)) break;  // (the phase before the first one counts as past)
        tc_fence_after();
        const float m_prev = h > 0 ? sh.m[row] : kNoReference;
        bool moved = false;
        float alpha = 1.f;
        auto new_reference = [&](float x_max) -> bool {  // true: it has moved (some row's of the warp)
          const bool grow = x_max > m_ref + kMaxGrowth;
          const float m_new = grow ? x_max + kHeadroom : m_ref;
          sh.m[row] = m_new;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.m_ready[w][quarter]);
          if (__builtin_expect(!__any_sync(0xffffffffu, grow), 1)) return false;
          moved = true;
          alpha = ex2(m_ref - m_new);
          l_run *= alpha;
          m_ref = m_new;
          return true;
        };
        uint64_t sums[2] = {0ull, 0ull};
        const int keys = h == n_steps - 1 ? ends : kKeyStep;
        // (A way of its own for up to 32 keys took 12 heads x 32760 over 16 from 54 us to 47, and over 128, 512 from 54.7 to 56.6, 108 to 111: code that is in the way.)
        if (__builtin_expect(keys < kKeyStep, 0)) {  // scores behind the last key
          int k = keys;
#pragma unroll 1
          for (; k & 7; ++k) tmem_st1(s_at + k, 0xff800000u);
#pragma unroll 1
          for (; k < kKeyStep; k += 8) tmem_st8_fill(s_at + k, 0xff800000u);
          tmem_wait_st();
        }
        uint32_t s[128], pk[32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(s_at + q * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[q * 32]));
        l_run *= ex2(m_ref - m_prev);
        m_ref = m_prev;
        tmem_wait_ld();
        arrive(&sh.s_free[w]);
        uint64_t neg_m2;
        bool again = false;
#pragma unroll 1
        do {  // (the first weights with the reference before, while the maximum is found)
          neg_m2 = pack_f32x2(-m_ref, -m_ref);
          sums[0] = sums[1] = 0ull;
          exp32<false>(&s[0], c2, neg_m2, &pk[0], sums);
          const float x_max = fmaxf(max64(&s[0]), max64(&s[64])) * c;
          again = !again && new_reference(x_max);
        } while (__builtin_expect(again, 0));
        const bool p_done = g < 2 || mbar_test_wait(&sh.pv_done[w], ((g - 2) >> 1) & 1);
        exp32<false>(&s[32], c2, neg_m2, &pk[16], sums);
        if (__builtin_expect(!__all_sync(0xffffffffu, p_done), 0)) wait(&sh.pv_done[w], ((g - 2) >> 1) & 1);
        tc_fence_after();
        tmem_st32(p_at, pk);
        exp32<false>(&s[64], c2, neg_m2, &pk[0], sums);
        exp32<false>(&s[96], c2, neg_m2, &pk[16], sums);
        tmem_st32(p_at + 32, pk);
        float s0, s1, s2, s3;
        unpack_f32x2(sums[0], s0, s1);
        unpack_f32x2(sums[1], s2, s3);
        l_run += (s0 + s1) + (s2 + s3);
        if (h >= n_steps - 2) {  // the row sum, by way of the other warpgroup to those who write
          const int at = n & 1;
          const uint32_t phase = (n >> 1) & 1;
          if ((h < n_steps - 1 || h == 0) && !wait(&sh.l_read[at], phase ^ 1)) break;  // (the first one's place has been free before)
          if (h == n_steps - 1) {
            float l = l_run;
            if (h > 0) {
              if (!wait(&sh.l_ready[at][quarter], phase)) break;
              l = fmaf(sh.l[at][row], ex2(m_prev - m_ref), l);
            }
            if (__builtin_expect(steps.w, 1)) {
              sh.l[at][row] = l == 0.f ? 0.f : reciprocal(l);
              if (p.lse != nullptr && row < x->tokens * p.G) *lse_of(x->row, x->h, row) = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * 0.6931471805599453f;
            } else {
              __stcg(&p.part_l[(2 * blockIdx.x + (steps.z == 0 ? 1 : 0)) * 128 + row], make_float2(l, m_ref));
            }
          } else {
            sh.l[at][row] = l_run;
          }
          __syncwarp();
          if (lane == 0 && (h < n_steps - 1 || h == 0)) mbar_arrive(&sh.l_ready[at][quarter]);
          if (lane == 0 && h == n_steps - 1) mbar_arrive(&sh.l_final[at]);
        }
        if (!ok) break;
        if (__builtin_expect(moved && h > 0, 0)) {
          // O changes scale: the products of the steps before have to be complete
          if (!wait(&sh.pv_done[w ^ 1], ((g - 1) >> 1) & 1)) break;
          tc_fence_after();
          const uint64_t alpha2 = pack_f32x2(alpha, alpha);
#pragma unroll 1
          for (int ch = 0; ch < 8; ++ch) {
            uint32_t v[16];
            tmem_ld16(o_addr + ch * 16, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              float lo, hi;
              unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), alpha2), lo, hi);
              v[i] = __float_as_uint(lo);
              v[i + 1] = __float_as_uint(hi);
            }
            tmem_st16(o_addr + ch * 16, v);
          }
        }
        tmem_wait_st();
        arrive(&sh.p_full[w]);
      }
      g0 += n_steps;
      done_with_part(n);
    }
  }

  // ------------------------------------------------------------------ tear-down
  __syncwarp();
  if (warp != kWarpK && lane == 0) mbar_arrive(&sh.finished);
  tc_fence_before();
  // Neither CTA of a pair leaves while the other one's products read its shared memory or arrivals are under way; after an abort copies in flight get time to
  // land (bounded: a copy takes microseconds).
  if (Pair) cluster_sync();
  else __syncthreads();
  int gave_up = *abort;
  if (Pair) gave_up |= (int)cluster_ld1(cluster_address(smem_u32(&sh.abort), rank ^ 1));
  if (gave_up) {
    const uint32_t since = clock();
    while ((uint32_t)clock() - since < 2000000u) {
    }
  }
  if (Pair) cluster_sync();
  else __syncthreads();
  if (warp == kWarpQK) {
    tc_fence_after();
    if (Pair) tmem_dealloc_pair(tmem, 512);
    else tmem_dealloc(tmem, 512);
  }
  // Shared tiles whose last part is here, by all threads: 16 dims of a row at a time.  (By the warpgroup that writes, as soon as a part was the last one, 4 heads x 300 over
  // 4000, 11 parts a tile, took 97 us, now 25.)
#pragma unroll 1
  for (int i = 0; i < (gave_up ? 0 : sh.n_merges); ++i) {
    const int4 x = sh.merges[i];
    const int row = tid & 127, tokens = x.y & 255, h = x.y >> 8;
    if (row >= tokens * p.G) continue;
    const int t = (int)(((uint32_t)row * p.inv_G) >> 16);
    uint16_t *const to = p.O + (long long)(x.x + t) * p.qt + (long long)(h * p.G + row - t * p.G) * p.qh;
#pragma unroll 1
    for (int d = (tid >> 7) * 32, end = d + 32; d < end; d += 16) {
      float m = kNoReference, l = 0.f, v[16] = {};
#pragma unroll 2
      for (int k = 0; k < x.w; ++k) {
        const int at = 2 * ((x.z + k) * kCtas + rank) + (k == 0 ? 1 : 0);
        const float2 lm = __ldcg(&p.part_l[at * 128 + row]);
        const float4 *src = &p.parts[(size_t)(at * 32 + (d >> 2)) * 128 + row];
        const float4 z0 = __ldcg(src), z1 = __ldcg(src + 128), z2 = __ldcg(src + 256), z3 = __ldcg(src + 384);
        const float top = fmaxf(m, lm.y), a = ex2(m - top), f = ex2(lm.y - top), z[16] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w, z2.x, z2.y, z2.z, z2.w, z3.x, z3.y, z3.z, z3.w};
        m = top;
        l = fmaf(l, a, lm.x * f);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = fmaf(z[j], f, v[j] * a);
      }
      const float inv = l == 0.f ? 0.f : reciprocal(l);
      uint32_t y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = pack_bf16x2(v[2 * j] * inv, v[2 * j + 1] * inv);
      *reinterpret_cast<uint4 *>(to + d) = make_uint4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<uint4 *>(to + d + 8) = make_uint4(y[4], y[5], y[6], y[7]);
      if (d == 0 && p.lse != nullptr) *lse_of(x.x, h, row) = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    }
  }
  if (sh.abort && tid == 0) {
    atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
#pragma unroll 1
    for (int i = sh.shared_parts; i < sh.n_owed; ++i) {  // what this CTA still owes to shared tiles: no numbers
      const int4 x = sh.owed[i];
#pragma unroll 1
      for (int r = 0; r < 128; ++r) __stcg(&p.part_l[x.x * 128 + r], make_float2(__uint_as_float(0x7fc00000u), 0.f));
      __threadfence();
      if (atomicAdd(&p.arrivals[x.y], 1) == x.z - 1) p.arrivals[x.y] = 0;
    }
  }
}

}  // namespace

cudaError_t launch_cross_tiles(const CrossGeom &g, const CacheIndex &ix, const CrossWorkspace &w, const void *Q, const void *K, const void *V, void *O,
                               float *lse, bool pair, cudaStream_t s, int *launches) {
  CUtensorMap mq, mk, mv, mo;
  if (!make_query_map(&mq, Q, g) || !make_query_map(&mo, O, g) || !make_states_map(&mk, K, g, pair ? kKeyStep / 2 : kKeyStep, 2) ||
      !make_states_map(&mv, V, g, kKeyStep, pair ? 1 : 2))
    return cudaErrorInvalidValue;
  CrossParams p = {};
  p.ix = ix;
  p.arrivals = w.arrivals;
  p.parts = reinterpret_cast<float4 *>(w.parts);
  p.part_l = w.part_l;
  p.O = static_cast<uint16_t *>(O);
  p.lse = lse;
  p.qt = g.qt;
  p.qh = g.qh;
  p.Hq = g.Hq;
  p.Hkv = g.Hkv;
  p.G = g.G;
  p.inv_G = (65536u + g.G - 1) / g.G;
  p.scale_log2 = (float)(g.scale * 1.4426950408889634);
  p.test_skip = g.test_skip;
  auto *const kernel = pair ? cross_tile_kernel<true> : cross_tile_kernel<false>;
  cudaError_t e = allow_shared_memory(kernel, kSmem);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_pdl(kernel, dim3(kCacheCtas), dim3(kThreads), kSmem, s, Cluster{pair ? 2 : 1}, mq, mk, mv, mo, p);
}

}  // namespace heart
