// Cross attention for many query rows a sequence and key head, on the sm_100a tensor cores.
//
// A tile is 128 rows: 128 / G tokens of a sequence with the G query heads of one key head.  Keys are processed 128 at a time, one CTA an SM, two
// softmax warpgroups that take the CTA's key steps in turn, scores double-buffered in tensor memory; the reasons are those at the top of attn_tc.cu, and so
// are what bounds it (the tensor pipe 1024 clocks a step, the special-function units 1024, shared memory 1280) and the way two warpgroups agree on a
// row's reference.  What differs, since all rows of a tile see the same keys and these are few (a text: 512, four steps):
//   * The end of a tile is the common case.  A warpgroup of its own takes the sums out of tensor memory and writes the rows, straight from
//     registers (a thread has a row, 32 bytes a store), while the others are in the next tile's first steps.
//   * A tile's last step may have fewer than 128 keys: the products are cut to the next 16 keys (columns of the scores, steps of the values' product),
//     the softmax to the next 32; scores behind the last key become -inf, values of up to 15 rows behind it, which are anyone's, zeros in shared memory.
//   * There is no plan: all tiles of a sequence take the same number of steps, so a CTA finds its share of the line of all tiles' steps, (sequence, head,
//     tile, step), from the lengths alone, each beginning of a tile counted as kTileCost steps.
//     Parts of a tile go to the workspace; the CTA that brings the last one puts them together, in order: the result does not depend on which one
//     that is.
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

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kWarpQK = 8, kWarpV = 9, kWarpK = 10, kWarpPV = 11, kWarpOut = 12;
constexpr int kRegsSoftmax = 192, kRegsOut = 72, kRegsHelper = 56;  // 192 * 256 + 72 * 128 + 56 * 128 = the CTA's 512 x 128
static_assert(kRegsSoftmax * 256 + kRegsOut * 128 + kRegsHelper * 128 <= kThreads * 128, "registers at launch");
constexpr int kTileBytes = 32768;  // 128 rows x 128 dims: [2 dim halves][128 rows][64] bf16, 128-byte swizzle
constexpr int kTileCost = 1;       // of a tile besides its steps, in steps
constexpr int kWholeSteps = 8;     // tiles of no more steps are not shared
constexpr int kMaxParts = 12;      // of a tile, about
constexpr int kPartRing = 4;
constexpr int kReaders = 15;       // of announced parts: softmax and writing warps, issuers, V producer
constexpr float kNoReference = -3.0e38f;
constexpr float kHeadroom = 16.f, kMaxGrowth = 8.f;  // see attn_tc.cu

// Part of a tile that a CTA takes: steps a .. b - 1.
struct Part {
  int row, tokens, h;     // first packed row, tokens, key head
  int key, len, steps;    // first row of its keys, how many, in steps
  int a, b;               // b < 0: no part left
  int c0, parts;          // first CTA with a part of the tile, and how many there are
  int pad[2];
};
static_assert(sizeof(Part) % 16 == 0, "copied by words");

// Where a CTA is in the line of all tiles' costs.
struct Walk {
  Sequence q;
  int s, h, tile, off;  // off: what of the tile's cost lies before the share
  long long u, end, share;
  bool whole;           // tiles are not shared: a CTA takes those that begin in its share
};

struct CrossShared {
  uint64_t q_full[2], k_full[2], v_full[2];
  uint64_t v_ready[2];     // V_g has nothing behind its last key that a product reads
  uint64_t s_full[2], s_free[2], p_full[2], pv_done[2], m_ready[2][4];  // as in attn_tc.cu
  uint64_t o_full[2], o_free;
  uint64_t part_full[kPartRing], part_empty[kPartRing];
  uint64_t drain[2];
  uint64_t stored, told;   // this CTA's part of a tile is in the workspace; it is the last one or not
  Part part[kPartRing];
  float m[2][128];         // references after step g
  float2 l[4][2][128];     // row sums and references: per part & 3 and warpgroup
  long long sums[kWarps];
  int longest[kWarps];
  Walk walk;
  Sequence found;          // the share's first sequence
  int found_s;
  long long found_at;      // cost before it
  uint32_t tmem_base;
  int shared_parts;        // parts of shared tiles that have been announced
  int last;
  int abort;
};
constexpr int kOffQ = 0, kOffK = 2 * kTileBytes, kOffV = 4 * kTileBytes, kOffShared = 6 * kTileBytes;
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
  bool wide;               // rows of O begin on 32 bytes
  int test_skip;           // test-hook builds only: CTA 0 leaves out its second copy of values
};

__device__ __forceinline__ void store32(uint16_t *to, const uint32_t *x, bool wide) {  // 32 bytes
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]),
                 "r"(x[6]), "r"(x[7])
                 : "memory");
  } else {
    *reinterpret_cast<uint4 *>(to) = make_uint4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<uint4 *>(to + 8) = make_uint4(x[4], x[5], x[6], x[7]);
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    cross_tile_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const CrossParams p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  CrossShared &sh = *reinterpret_cast<CrossShared *>(smem + kOffShared);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const CacheIndex &ix = p.ix;
  volatile int *abort = &sh.abort;

  // ------------------------------------------------------------------ set-up
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1);
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.v_ready[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], 4);
      mbar_init(&sh.p_full[i], 4);
      mbar_init(&sh.pv_done[i], 1);
      for (int q = 0; q < 4; ++q) mbar_init(&sh.m_ready[i][q], 1);
      mbar_init(&sh.o_full[i], 1);
      mbar_init(&sh.drain[i], 1);
    }
    for (int i = 0; i < kPartRing; ++i) {
      mbar_init(&sh.part_full[i], 1);
      mbar_init(&sh.part_empty[i], kReaders);
    }
    mbar_init(&sh.o_free, 4);
    mbar_init(&sh.stored, 4);
    mbar_init(&sh.told, 1);
    sh.abort = 0;
    sh.shared_parts = 0;
    mbar_fence_init();
  }
  if (warp == kWarpK && lane == 0) {
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  pdl_wait();
  pdl_launch_dependents();

  // ------------------------------------------------------------------ the CTA's share of the line
  const int tokens_per_tile = 128 / p.G;
  auto tiles_of = [&](const Sequence &q) { return (int)(((long long)q.n + tokens_per_tile - 1) / tokens_per_tile); };
  auto steps_of = [&](const Sequence &q) { return max((q.len + kKeyStep - 1) / kKeyStep, 1); };  // (one without any key: the rows are written)
  auto cost_of = [&](const Sequence &q) { return steps_of(q) + kTileCost; };
  {
    Sequence q = {0, 0, 0, 0};
    long long mine = 0, total = 0;
    int longest = 1;
    for (int i = tid; i < ix.S; i += kThreads) {
      const Sequence x = cross_sequence(ix, i);
      const int tiles = tiles_of(x), cost = cost_of(x);
      const long long all = (long long)tiles * cost * p.Hkv;
      if (i < kThreads) q = x, mine = all;
      if (tiles > 0) longest = max(longest, cost);
      total += all;
    }
    const long long first_mine = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 0) sh.sums[warp] = total, sh.longest[warp] = longest;
    __syncthreads();
    total = 0;
    for (int i = 0; i < kWarps; ++i) {
      total += sh.sums[i];
      longest = max(longest, sh.longest[i]);
    }
    const bool whole = longest <= kWholeSteps + kTileCost;
    const long long share = max((total + gridDim.x - 1) / gridDim.x, whole ? 1LL : (long long)(longest + kMaxParts - 1) / kMaxParts);
    const long long u0 = blockIdx.x * share, u1 = min(total, u0 + share);
    if (u0 >= u1) return;
    if (tid == 0) sh.walk.end = u1, sh.walk.share = share, sh.walk.whole = whole;
    long long before = 0;
    mine = first_mine;
    for (int base = 0; base < ix.S; base += kThreads) {
      if (base > 0) {
        mine = 0;
        if (base + tid < ix.S) {
          q = cross_sequence(ix, base + tid);
          mine = (long long)tiles_of(q) * cost_of(q) * p.Hkv;
        }
      }
      long long upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      __syncthreads();
      if (lane == 31) sh.sums[warp] = upto;
      __syncthreads();
      long long at = before + upto - mine, all = 0;
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) at += sh.sums[i];
        all += sh.sums[i];
      }
      if (at <= u0 && u0 < at + mine) {
        sh.found = q;
        sh.found_s = base + tid;
        sh.found_at = at;
      }
      before += all;
      if (before > u0) break;
    }
  }
  if (warp == kWarpQK) {
    tmem_alloc(&sh.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;

  // Bounded waits of a whole warp; ok turns false when one runs out or the CTA aborts.
  bool ok = true;
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    uint32_t since = 0;
#pragma unroll 1
    while (__builtin_expect(!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)), 0)) {
      const uint32_t now = clock() | 1u;
      if (since == 0) since = now;
      if (__any_sync(0xffffffffu, *abort != 0 || now - since > (uint32_t)kWaitLimitCycles)) {
        *abort = 1;
        return ok = false;
      }
    }
    return ok;
  };
  // The announced part n; nullptr: none left (or abort).
  auto part_at = [&](int n) -> const Part * {
    if (!wait(&sh.part_full[n % kPartRing], (n / kPartRing) & 1)) return nullptr;
    const Part *x = &sh.part[n % kPartRing];
    return x->b < 0 ? nullptr : x;
  };
  auto done_with_part = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_empty[n % kPartRing]);
  };
  // Keys of a part's last step: fewer than 128 if that is the tile's last one.
  auto last_keys = [&](const Part *x) { return x->b < x->steps ? kKeyStep : x->len - (x->steps - 1) * kKeyStep; };
  auto settle = [&](uint64_t *bar, uint32_t parity) {
    const uint32_t t0 = clock();
    while (!mbar_try_wait(bar, parity) && (uint32_t)clock() - t0 < 40000000u) {
    }
  };
  auto settle_pair = [&](uint64_t *bar, int issued) {  // the last two of `issued` copies on a pair of barriers
#pragma unroll 1
    for (int i = issued > 2 ? issued - 2 : 0; i < issued; ++i) settle(&bar[i & 1], (i >> 1) & 1);
  };
  auto desc_at = [](uint64_t desc, uint32_t off16) -> uint64_t {
    return (desc & 0xffffffff00000000ull) | (uint32_t)((uint32_t)desc + off16);
  };
  auto drain_products = [&](bool leader, uint64_t *bar) {
    if (!*abort) return;
    if (leader) tc_commit(bar);
    __syncwarp();
    settle(bar, 0);
  };
  auto load_tile = [&](unsigned char *dst, const CUtensorMap *map, uint64_t *bar, int row, int h) {
    if (lane == 0) {
      mbar_expect_tx(bar, kTileBytes);
      tma_load_5d(dst, map, bar, 0, row, 0, h, 0);
    }
  };
  // ------------------------------------------------------------------ the CTA's parts, in order (by one thread, in shared memory)
  auto walk_begins = [&](Walk &w) {
    w.q = sh.found;
    w.s = sh.found_s;
    const int tiles = tiles_of(w.q), cost = cost_of(w.q);
    w.u = blockIdx.x * w.share;
    const long long rest = w.u - sh.found_at;
    const long long at = rest / cost;  // tile of all heads
    w.off = (int)(rest - at * cost);
    w.h = (int)(at / tiles);
    w.tile = (int)(at - (long long)w.h * tiles);
  };
  auto walk_on = [&](Walk &w) {  // to the next tile, whose cost begins at u
    w.off = 0;
    if (++w.tile < tiles_of(w.q)) return;
    w.tile = 0;
    if (++w.h < p.Hkv) return;
    w.h = 0;
    do w.q = cross_sequence(ix, ++w.s);
    while (w.q.n == 0 && w.s + 1 < ix.S);
  };
  // The part at w, behind which w then is; false: none left.
  auto next_part = [&](Walk &w, Part &x) {
    if (w.whole && w.off > 0) {
      w.u += cost_of(w.q) - w.off;
      if (w.u < w.end) walk_on(w);
    }
    x.b = -1;
    if (w.u >= w.end) return false;
    const int steps = steps_of(w.q);
    const int a = max(w.off - kTileCost, 0);
    const int b = w.whole ? steps : (int)min((long long)steps, w.off + (w.end - w.u) - kTileCost);
    if (b <= a) return false;  // (the share ends before the tile's first step)
    x.row = w.q.row + w.tile * tokens_per_tile;
    x.tokens = min(tokens_per_tile, w.q.n - w.tile * tokens_per_tile);
    x.h = w.h;
    x.key = w.q.key;
    x.len = w.q.len;
    x.steps = steps;
    x.a = a;
    x.b = b;
    const long long first = w.u - w.off + kTileCost;
    x.c0 = blockIdx.x;
    x.parts = 1;
    if (b - a < steps) {
      x.c0 = (int)(first / w.share);
      x.parts = (int)((first + steps - 1) / w.share) - x.c0 + 1;
    }
    w.u += b + kTileCost - w.off;
    if (w.u < w.end) walk_on(w);
    return true;
  };

  // ------------------------------------------------------------------ roles
  if (warp >= kWarpOut) {
    setmaxnreg_dec<kRegsOut>();
  } else if (warp >= kWarpQK) {
    setmaxnreg_dec<kRegsHelper>();
  }
  if (warp == kWarpK) {
    // ===== the CTA's parts; K and Q producer
    if (lane == 0) walk_begins(sh.walk);
    auto announce = [&](int m) {
      if (m >= kPartRing && !wait(&sh.part_empty[m % kPartRing], (m / kPartRing - 1) & 1)) return false;
      Part &x = sh.part[m % kPartRing];
      if (lane == 0) {
        next_part(sh.walk, x);
        mbar_arrive(&sh.part_full[m % kPartRing]);
      }
      __syncwarp();
      return x.b >= 0;
    };
    int g = 0, n = 0;
    bool any = announce(0);
#pragma unroll 1
    for (; ok && any; ++n) {
      const Part &x = sh.part[n % kPartRing];  // (this warp alone writes the ring)
      const int a = x.a, b = x.b, h = x.h, key = x.key, row = x.row;
#pragma unroll 1
      for (int i = a; i < b; ++i, ++g) {
        if (g >= 2 && !wait(&sh.s_full[g & 1], ((g - 2) >> 1) & 1)) break;
        load_tile(smem + kOffK + (g & 1) * kTileBytes, &map_k, &sh.k_full[g & 1], key + i * kKeyStep, h);
        if (i == a && lane == 0) {  // (the scores of step g - 2 are complete, and with them those of part n - 2: its Q has been read)
          unsigned char *q = smem + kOffQ + (n & 1) * kTileBytes;
          mbar_expect_tx(&sh.q_full[n & 1], 2 * (128 / p.G * p.G) * 128);
          tma_load_5d(q, &map_q, &sh.q_full[n & 1], 0, 0, row, 0, h);
          tma_load_5d(q + kTileBytes / 2, &map_q, &sh.q_full[n & 1], 0, 0, row, 1, h);
        }
        __syncwarp();
      }
      if (ok) any = announce(n + 1);
    }
    if (*abort) {
      settle_pair(sh.k_full, g);
      settle_pair(sh.q_full, n);  // (n counts a part that was broken off too: its Q came with its first step, or not at all)
    }
  } else if (warp == kWarpV) {
    // ===== V producer
    int g = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int a = x->a, b = x->b, h = x->h, key = x->key, ends = last_keys(x);
      done_with_part(n);
#pragma unroll 1
      for (int i = a; i < b; ++i, ++g) {
        const int at = g & 1;
        if (g >= 2 && !wait(&sh.pv_done[at], ((g - 2) >> 1) & 1)) break;
        unsigned char *const to = smem + kOffV + at * kTileBytes;
#ifdef HEART_TEST_HOOKS
        if (!(p.test_skip && blockIdx.x == 0 && g == 1))
#endif
        load_tile(to, &map_v, &sh.v_full[at], key + i * kKeyStep, h);
        const int keys = i == b - 1 ? ends : kKeyStep;
        if ((keys & 15) || keys == 0) {  // rows that a product reads behind the last key
          if (!wait(&sh.v_full[at], (g >> 1) & 1)) {
            ++g;
            break;
          }
          const int out = keys == 0 ? 16 : 16 - (keys & 15);
          for (int j = lane; j < out * 16; j += 32)
            sts_u4(smem_u32(to) + ((j >> 3) & 1) * (kTileBytes / 2) + (keys + (j >> 4)) * 128 + (j & 7) * 16, make_uint4(0u, 0u, 0u, 0u));
          async_proxy_fence();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.v_ready[at]);
      }
    }
    if (*abort) settle_pair(sh.v_full, g);
  } else if (warp == kWarpQK) {
    // ===== issuer of the score products
    const uint64_t q_desc = smem_desc_sw128(smem_u32(smem + kOffQ), 16, 1024);
    const uint64_t k_desc = smem_desc_sw128(smem_u32(smem + kOffK), 16, 1024);
    const bool leader = elect_one();
    uint32_t g = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int n_steps = x->b - x->a, ends = last_keys(x);
      done_with_part(n);
      wait(&sh.q_full[n & 1], (n >> 1) & 1);
      const uint64_t qd = desc_at(q_desc, (n & 1) * (kTileBytes >> 4));
#pragma unroll 1
      for (int i = 0; i < n_steps; ++i, ++g) {  // S_g = Q K_g^T
        const uint32_t b = g & 1;
        if (g >= 2) wait(&sh.s_free[b], ((g - 2) >> 1) & 1);
        if (!wait(&sh.k_full[b], (g >> 1) & 1)) break;
        tc_fence_after();
        if (leader) {
          const uint64_t kd = desc_at(k_desc, b * (kTileBytes >> 4));
          const int keys = i == n_steps - 1 ? max((ends + 15) & ~15, 16) : kKeyStep;
          const uint32_t idesc = idesc_bf16_f32(128, 0, false, false) | (uint32_t)(keys >> 3) << 17;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            mma_ss(tmem + 128 + b * 128, desc_at(qd, (ks >> 2) * 1024 + (ks & 3) * 2), desc_at(kd, (ks >> 2) * 1024 + (ks & 3) * 2), idesc, ks > 0 ? 1u : 0u);
          tc_commit(&sh.s_full[b]);
        }
        __syncwarp();
      }
    }
    drain_products(leader, &sh.drain[0]);
  } else if (warp == kWarpPV) {
    // ===== issuer of the value products
    constexpr uint32_t idesc = idesc_bf16_f32(128, 128, false, true);
    const uint64_t v_desc = smem_desc_sw128(smem_u32(smem + kOffV), kTileBytes / 2, 1024);
    const bool leader = elect_one();
    uint32_t g = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int n_steps = x->b - x->a, ends = last_keys(x);
      done_with_part(n);
      if (n > 0) wait(&sh.o_free, (n - 1) & 1);
#pragma unroll 1
      for (int i = 0; i < n_steps; ++i, ++g) {  // O (+)= P_g V_g
        const uint32_t b = g & 1;
        wait(&sh.v_full[b], (g >> 1) & 1);
        wait(&sh.v_ready[b], (g >> 1) & 1);
        if (!wait(&sh.p_full[b], (g >> 1) & 1)) break;
        tc_fence_after();
        if (leader) {
          const uint64_t vd = desc_at(v_desc, b * (kTileBytes >> 4));
          const int ks_end = i == n_steps - 1 ? max((ends + 15) >> 4, 1) : 8;
          if (ks_end == 8) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) mma_ts(tmem, tmem + 384 + b * 64 + ks * 8, desc_at(vd, ks * 128), idesc, (i > 0 || ks > 0) ? 1u : 0u);
          } else {
#pragma unroll 1
            for (int ks = 0; ks < ks_end; ++ks) mma_ts(tmem, tmem + 384 + b * 64 + ks * 8, desc_at(vd, ks * 128), idesc, (i > 0 || ks > 0) ? 1u : 0u);
          }
          if (i == n_steps - 1) tc_commit(&sh.o_full[n & 1]);
          tc_commit(&sh.pv_done[b]);
        }
        __syncwarp();
      }
    }
    drain_products(leader, &sh.drain[1]);
  } else if (warp >= kWarpOut) {
    // ===== output: thread = one row
    const uint32_t quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t o_addr = tmem + (quarter << 21);
    const int token = (int)(((uint32_t)row * p.inv_G) >> 16);
    uint32_t g_end = 0, n_stored = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int n_steps = x->b - x->a, n_rows = x->tokens * p.G, c0 = x->c0, parts = x->parts, first_row = x->row, h = x->h;
      const bool all = n_steps == x->steps, begins = x->a == 0;
      done_with_part(n);
      g_end += n_steps;
      if (!wait(&sh.o_full[n & 1], (n >> 1) & 1)) break;
      tc_fence_after();
      const uint32_t w_last = (g_end - 1) & 1;
      const float2 last = sh.l[n & 3][w_last][row];
      float l = last.x, m = last.y;
      if (n_steps > 1) {
        const float2 other = sh.l[n & 3][w_last ^ 1][row];
        l += other.x * ex2(other.y - m);
      }
      uint16_t *const o_row = p.O + (long long)(first_row + token) * p.qt + (long long)(h * p.G + row - token * p.G) * p.qh;
      const bool real = row < n_rows;
      auto write32 = [&](const uint32_t (&v)[32], int d, float inv) {
        const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float a0, a1;
            unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[k * 16 + 2 * i]), __uint_as_float(v[k * 16 + 2 * i + 1])), inv2), a0, a1);
            y[i] = pack_bf16x2(a0, a1);
          }
          if (real) store32(o_row + d + k * 16, y, p.wide);
        }
      };
      const int slot = 2 * blockIdx.x + (begins ? 1 : 0);
      float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t v[32];
        tmem_ld32(o_addr + c * 32, v);
        tmem_wait_ld();
        if (c == 3) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.o_free);
        }
        if (all) {
          write32(v, c * 32, inv);
        } else if (real) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            __stcg(&p.parts[((size_t)slot * 32 + c * 8 + i) * 128 + row],
                   make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3])));
        }
      }
      bool write = all;
      if (!all) {
        if (real) __stcg(&p.part_l[slot * 128 + row], make_float2(l, m));
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.stored);
        if (quarter == 0) {
          if (!wait(&sh.stored, n_stored & 1)) break;
          if (lane == 0) {
            __threadfence();  // (of what the warpgroup has stored, which the barrier has shown this thread)
            const bool is_last = atomicAdd(&p.arrivals[c0], 1) == parts - 1;
            if (is_last) p.arrivals[c0] = 0;
            sh.last = is_last;
            ++sh.shared_parts;
            __threadfence();
            mbar_arrive(&sh.told);
          }
          __syncwarp();
        }
        if (!wait(&sh.told, n_stored & 1)) break;
        ++n_stored;
        write = sh.last != 0;
        if (write && real) {
          auto place = [&](int i) { return 2 * (c0 + i) + (i == 0 ? 1 : 0); };
          m = kNoReference;
          l = 0.f;
#pragma unroll 4
          for (int i = 0; i < parts; ++i) m = fmaxf(m, __ldcg(&p.part_l[place(i) * 128 + row]).y);
#pragma unroll 4
          for (int i = 0; i < parts; ++i) {
            const float2 lm = __ldcg(&p.part_l[place(i) * 128 + row]);
            l = fmaf(lm.x, ex2(lm.y - m), l);
          }
          inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0u;
#pragma unroll 1
            for (int i = 0; i < parts; ++i) {
              const float f = ex2(__ldcg(&p.part_l[place(i) * 128 + row]).y - m);
              const float4 *src = &p.parts[((size_t)place(i) * 32 + c * 8) * 128 + row];
              float4 y[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) y[k] = __ldcg(src + k * 128);
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                v[4 * k] = __float_as_uint(fmaf(y[k].x, f, __uint_as_float(v[4 * k])));
                v[4 * k + 1] = __float_as_uint(fmaf(y[k].y, f, __uint_as_float(v[4 * k + 1])));
                v[4 * k + 2] = __float_as_uint(fmaf(y[k].z, f, __uint_as_float(v[4 * k + 2])));
                v[4 * k + 3] = __float_as_uint(fmaf(y[k].w, f, __uint_as_float(v[4 * k + 3])));
              }
            }
            write32(v, c * 32, inv);
          }
        }
      }
      if (write && real && p.lse != nullptr)
        p.lse[(long long)(first_row + token) * p.Hq + h * p.G + row - token * p.G] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
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
      if (lane == 0) mbar_arrive(bar);
    };
    uint32_t g0 = 0;  // key steps before the present part
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr) break;
      const int n_steps = x->b - x->a, ends = last_keys(x);
      done_with_part(n);
      float m_ref = kNoReference, l_run = 0.f;
#pragma unroll 1
      for (int h = (w ^ g0) & 1; h < n_steps; h += 2) {
        const uint32_t g = g0 + h;
        if (g > 0 && !wait(&sh.m_ready[w ^ 1][quarter], ((g - 1) >> 1) & 1)) break;
        if (!wait(&sh.s_full[w], (g >> 1) & 1)) break;
        tc_fence_after();
        const float m_prev = h > 0 ? sh.m[w ^ 1][row] : kNoReference;
        bool moved = false;
        float alpha = 1.f;
        auto new_reference = [&](float x_max) -> bool {  // true: it has moved (some row's of the warp)
          const bool grow = x_max > m_ref + kMaxGrowth;
          const float m_new = grow ? x_max + kHeadroom : m_ref;
          sh.m[w][row] = m_new;
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
        if (keys == kKeyStep) {
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
        } else {
          // 32 keys at a time: once for the maximum, once for the weights
          uint32_t s[32], pk[16];
          auto load = [&](int k0) {
            tmem_ld32(s_at + k0, s);
            tmem_wait_ld();
            if (k0 + 32 > keys) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (k0 + i >= keys) s[i] = 0xff800000u;
            }
          };
          l_run *= ex2(m_ref - m_prev);
          m_ref = m_prev;
          float x_max = -INFINITY;
          const int end = max(keys, 1);
#pragma unroll 1
          for (int k0 = 0; k0 < end; k0 += 32) {
            load(k0);
#pragma unroll
            for (int i = 0; i < 32; i += 2) x_max = fmax3(x_max, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
          }
          new_reference(x_max * c);
          if (g >= 2 && !wait(&sh.pv_done[w], ((g - 2) >> 1) & 1)) break;
          tc_fence_after();
          const uint64_t neg_m2 = pack_f32x2(-m_ref, -m_ref);
#pragma unroll 1
          for (int k0 = 0; k0 < end; k0 += 32) {
            load(k0);
            exp32<false>(s, c2, neg_m2, pk, sums);
            tmem_st16(p_at + (k0 >> 1), pk);
          }
          arrive(&sh.s_free[w]);
        }
        float s0, s1, s2, s3;
        unpack_f32x2(sums[0], s0, s1);
        unpack_f32x2(sums[1], s2, s3);
        l_run += (s0 + s1) + (s2 + s3);
        if (h >= n_steps - 2) sh.l[n & 3][w][row] = make_float2(l_run, m_ref);
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
    }
  }

  // ------------------------------------------------------------------ tear-down
  tc_fence_before();
  __syncthreads();
  if (warp == kWarpQK) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (sh.abort && tid == 0) {
    atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
    // what this CTA still owes to shared tiles: no numbers
    walk_begins(sh.walk);
    Part &x = sh.part[0];
    for (int i = 0; next_part(sh.walk, x);) {
      if (x.parts == 1 || i++ < sh.shared_parts) continue;
      const int slot = 2 * blockIdx.x + (x.a == 0 ? 1 : 0);
      for (int r = 0; r < 128; ++r) __stcg(&p.part_l[slot * 128 + r], make_float2(__uint_as_float(0x7fc00000u), 0.f));
      __threadfence();
      if (atomicAdd(&p.arrivals[x.c0], 1) == x.parts - 1) p.arrivals[x.c0] = 0;
    }
  }
}

}  // namespace

cudaError_t launch_cross_tiles(const CrossGeom &g, const CacheIndex &ix, const CrossWorkspace &w, const void *Q, const void *K, const void *V, void *O,
                               float *lse, cudaStream_t s, int *launches) {
  CUtensorMap mq, mk, mv;
  if (!make_query_map(&mq, Q, g) || !make_states_map(&mk, K, g, kKeyStep) || !make_states_map(&mv, V, g, kKeyStep)) return cudaErrorInvalidValue;
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
  p.wide = (reinterpret_cast<uintptr_t>(O) & 31u) == 0 && g.qt % 16 == 0 && g.qh % 16 == 0;
  p.test_skip = g.test_skip;
  cudaError_t e = allow_shared_memory(cross_tile_kernel, kSmem);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_pdl(cross_tile_kernel, dim3(kCacheCtas), dim3(kThreads), kSmem, s, mq, mk, mv, p);
}

}  // namespace heart
