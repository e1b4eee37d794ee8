// Attention over a paged cache for many query rows a sequence and key head, on the sm_100a tensor cores.
//
// A tile is 128 rows: 128 / G tokens of a sequence with the G query heads of one key head.  Keys are processed 128 at a time, one
// CTA an SM, two softmax warpgroups that take a tile's key steps (nearly) in turn, scores double-buffered in tensor memory; the
// reasons are those at the top of attn_tc.cu, and so are what bounds it (the tensor pipe 1024 clocks a step, the special-function
// units 1024, shared memory 1280) and the way two warpgroups agree on a row's reference.  What differs:
//   * Keys and values come page by page, 128 / page boxes for every 128 keys, with the page numbers fetched a step ahead.
//   * Rows see different keys.  Steps that some row does not see whole have a path of their own, outside of the loop over the steps:
//     hidden scores become -inf in tensor memory, and values that are not finite (what lies behind a sequence's end is anyone's) are
//     taken out of shared memory first, because the product reads them with weight 0; rows that do see such a value are marked.
//   * Tiles, of one key head after the other, are dealt in turn, so that the CTAs read the same keys at a time (12 x 32760 over themselves, 201 MB
//     of keys and values: 7.2 ms when every CTA had a run of tiles of its own, whose keys came from DRAM, 5.7 dealt; where they fit the L2 both
//     take the same time), but for the last one to two rounds of them: the steps of those, in one line, are cut into shares that
//     bring all CTAs to the same sum, so that the launch ends on all SMs at once whatever the lengths are.  The sum counts a tile's beginning
//     and end as four steps and a step that some row does not see whole as three (12 x 4680 over 32760, causal by frames, 770 us with
//     steps alone, now 738; 6 prompts x 24 heads 130, now 126; other weights near these give the same), unless the launch has less
//     than two tiles a CTA.  Parts of a tile go to the workspace; the CTA that brings the last one puts them together, in order: the
//     result does not depend on which one that is.
//
// e4m3 caches.  Converting keys and values to bf16 for 128 rows costs as many instructions as the softmax does.  Keys need none: a bf16 query has
// 8 significant bits and a code 4, so a query row, scaled by a power of two, is the sum of two rows of codes, to 2^-18 of its
// largest element, and two products with the keys' codes at twice the rate take the time of one in bf16.  Weights are
// not split that way (many keys of little weight each would be lost): values are converted by a fourth warpgroup, to f16, which takes one
// instruction for two codes, where bf16 takes nine for four (3900 clocks a step).  The keys' scales multiply the scores; the values' do not fit f16
// whatever they are, so a step's values are code * 2^(e - E), E the largest exponent of the step, and its weights
// 2^(score + E - m): the reference of a row is over score + E.  The sums, of 2^(score - m + E of the part's first step), take 2^(that - E) a
// step.
// That is right where exponents lie near each other.  Of the tokens that some row of a sequence sees those of a step may be kScaleSpan
// binades apart: a product of a weight and a scale then counts as zero only below 2^-23 of the row's largest (f16 has 2^-25, the largest is at 2^6 and
// more of the step's E).  From step to step E may move by kScaleRange, which costs nothing (the sums have 32 bits); but a value of zero, which has its
// step's E, is to raise no row's reference by more than kScaleSpan above what other steps have.  CTAs of the plan launch look at all scales, while one of them plans (the
// V producer, which has them at hand, sets the pace: looked at there, 12 heads x 4680 over 12 680 took 459 us instead of 378); a sequence and key head that is beyond these is
// done again by rows (cache_rows.cu), where a weight has its own token's scale: all of 12 heads x 4680 over 12 680 2.9 ms, one of them 0.2 ms.  The look and the second launch
// cost 2 to 4 us a call.
//
// Warp roles: 0-3, 4-7 softmax; 8 issues S = Q K^T; 9 copies V; 10 finds the CTA's parts and the pages of their steps, copies K and Q; 11
// issues O += P V; 12-15 (e4m3) convert.  Tensor memory: O (128 columns) | S[2] (2 x 128) | P[2] (2 x 64).
// Every wait is bounded; one that runs out raises the CTA's abort flag and the status word, and its roles stop.
//
// Times of long launches in this file were taken with pauses between the calls; back to back for a second, at the power limit, 40 heads x 4680 over 33k takes
// 3.3 ms where it has 2.8 to 2.9 then, and 12 x 4680 over 32760, causal by frames, 0.83 where it has 0.72.
#include <algorithm>

#include "cache.cuh"
#include "tc_ptx.cuh"
#include "tiles.cuh"

namespace heart {
using namespace tc;
namespace {

constexpr int kWarpQK = 8, kWarpV = 9, kWarpK = 10, kWarpPV = 11, kWarpConvert = 12;
constexpr int kTileBytes = 32768;  // 128 rows x 128 dims of bf16: [2 dim halves][128 rows][64], 128-byte swizzle
constexpr int kCodeBytes = 16384;  // the same as e4m3: [128 rows][128]
constexpr int kSteps = 16;         // key steps in flight (K is up to four steps ahead of the value products)
constexpr int kTileCost = 4, kMaskCost = 2;  // of a tile and of a step that some row does not see whole, in steps
constexpr int kPartRing = 8;       // parts are announced a part ahead
constexpr int kMaxParts = 12;      // of a tile, about
constexpr float kNoReference = -3.0e38f;
constexpr float kHeadroom = 16.f, kMaxGrowth = 8.f;  // see attn_tc.cu
constexpr float kHeadroomE4m3 = -6.f, kMaxGrowthE4m3 = 15.f;  // weights of f16: 2^6 where the reference moves, to 2^15
constexpr int kScaleSpan = 8, kScaleRange = 40;  // see above
constexpr int kNoValue = 17, kNoValueAs = 97;    // scale bytes up to this, of values below 2^-101, count as zeros; the E (as a byte) of a step of such ones
constexpr uint32_t kShortWait = 500;
constexpr int kRowsAtOnce = 4;  // of queries that are split

// A tile of a head as the plan kernel writes it.
struct Tile {
  int s, row, tokens, p0;         // sequence; first packed row; new tokens; position of the first
  int len, sinks, first, steps;   // tokens of the sequence; its key steps (see Span)
  int every_low, every_end;       // all rows see the keys every_low .. every_end - 1 (and of the sinks those before every_end)
  int some_low, some_end;         // some row sees them
  int extra;                      // what else it costs, in steps
};
constexpr int kTileWords = sizeof(Tile) / 4;
static_assert(sizeof(Tile) == kTileRecord, "the workspace has room for it");

// Part of a tile that a CTA takes: steps a .. b - 1 for key head h.
struct Part {
  Tile t;
  int h, a, b;       // b < 0: no part left
  int c0, parts;     // first CTA with a part of the tile, and how many there are
  int pad[3];
};
constexpr int kPartWords = sizeof(Part) / 4;
static_assert(kPartWords <= 32, "lanes copy words");

// A key step of a CTA, some steps ahead of its use.
struct Step {
  int key, seen, h, flags;  // first key; e4m3: see kStepUnseen; key head
  int page[8];
};
constexpr int kStepMasked = 1, kStepEnd = 2;  // some row does not see all of its keys; no step left
constexpr uint32_t kStepUnseen = 1u << 31;    // no row of the tile sees its keys before bits 8-15 (but for the sinks), nor those from bits 0-7 on

template <bool E4m3>
struct Layout {
  static constexpr int kThreads = E4m3 ? 512 : 384;
  static constexpr int kRegsSoftmax = E4m3 ? 192 : 224, kRegsHelper = 56, kRegsConvert = 72;  // sums: the registers at launch
  static constexpr int kReaders = E4m3 ? 15 : 11;  // of announced parts: softmax warps, issuers, V producer, converters
  static constexpr int kKey = E4m3 ? kCodeBytes : kTileBytes;
  // Q, K, V (of which the products read), codes of V
  static constexpr int kOffQ = 0, kOffK = 2 * kTileBytes, kOffV = kOffK + 2 * kKey, kOffCodes = kOffV + 2 * kTileBytes;
  static constexpr int kOffShared = kOffCodes + (E4m3 ? 2 * kCodeBytes : 0);
};

struct TileShared {
  uint64_t q_full[2], k_full[2], v_full[2];
  uint64_t q_ready[2];     // e4m3: Q as codes
  uint64_t v_ready[2];     // e4m3: V_g converted; bf16: V_g has nothing in it that is not finite, if its step is masked
  uint64_t codes_free[2];  // e4m3: the codes of V_g have been read
  uint64_t s_full[2], s_free[2], p_full[2], pv_done[2], m_ready[2][4];  // as in attn_tc.cu
  uint64_t o_full[2], o_free, out_done[2];
  uint64_t part_full[kPartRing], part_empty[kPartRing];
  uint64_t step_full[kSteps];
  uint64_t scales_full[8];  // e4m3: the factors of a step's keys are there
  uint64_t drain[2];
  uint64_t stored[2], told[2];  // a warpgroup's part of a tile is in the workspace; it is the last one or not
  Part part[kPartRing];
  Part written[2][8];        // the part to write, per softmax warp
  Step step[kSteps];
  float m[2][128];           // references after step g
  float2 l[4][2][128];       // row sums and references: per part & 3 and warpgroup (a warpgroup may be two short parts ahead of one that writes)
  alignas(16) float k_scale[8][128];  // e4m3, by g & 7
  uint8_t v_scale[8][128];            // scale bytes, 0: nothing
  int first_top[4];                   // the largest one of the first step, per part & 3
  int top[8];                         // the largest
  float q_scale[2][128];     // e4m3: what the scores of a row are to be multiplied by
  alignas(16) uint8_t zeros[128];     // e4m3: what the codes of a token count as that is none
  alignas(16) uint32_t bad[8][4];     // e4m3: keys that are not finite, by g & 7
  alignas(16) uint8_t not_finite[4][128];  // bf16: rows that see a value that is not finite, per part & 3
  uint32_t tmem_base;
  int last[2];
  int abort;
};
template <bool E4m3>
constexpr int kSmem = Layout<E4m3>::kOffShared + sizeof(TileShared);
static_assert(kSmem<true> <= 232448 && kSmem<false> <= 232448, "shared memory of an SM");

struct TileParams {
  CacheIndex ix;
  const Tile *tiles;
  const long long *first;  // [tiles] cost of what is before a tile of a head, in steps
  const int *head;         // number of tiles of a head, rounds of tiles that are dealt
  const long long *cuts;   // [CTAs + 1] where the shares of what follows begin, counted from the first tile that is not dealt
  int32_t *arrivals;
  float4 *parts;           // [2 * CTAs][32][128]: four dims of a row
  float2 *part_l;          // [2 * CTAs][128]
  uint16_t *O;
  float *lse;
  const uint8_t *k_scale, *v_scale;
  long long qt, qh;
  int Hq, Hkv, G;
  uint32_t inv_G;          // row / G = row * inv_G >> 16 for the rows of a tile
  float scale_log2;
  int test_skip;           // test-hook builds only: CTA 0 leaves out its second copy of values
  uint8_t *redo;           // see CacheWorkspace
  int *any_redo;
  __device__ __forceinline__ int token_of(int row) const { return (int)(((uint32_t)row * inv_G) >> 16); }
};

// D[tmem] (+)= A[smem] * B[smem], e4m3
__device__ __forceinline__ void mma_ss_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor for kind::f16 with f16 A/B and fp32 accumulator.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool a_mn_major, bool b_mn_major) {
  return (1u << 4) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__host__ __device__ constexpr uint32_t idesc_e4m3_f32(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);  // D f32, A and B e4m3 (0), K-major
}
__device__ __forceinline__ uint2 lds_u2(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts_u1(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
// Zero as long as all of the bf16 numbers so far are finite, NaN from the first one on that is not: 0 * x + sum.
__device__ __forceinline__ uint32_t add_zero_times(const uint4 &x, uint32_t sum) {
  auto add = [&](uint32_t w) { asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(w), "r"(0u)); };
  add(x.x), add(x.y), add(x.z), add(x.w);
  return sum;
}

// ---------------------------------------------------------------------- plan
// The scales of the values that the rows of a sequence see, for a key head: 1 if they are further apart than the tile kernel holds (see the
// top of the file).  2^warps_log2 warps a sequence and key head, or `ctas` CTAs each, a lane 16 tokens, eight lanes a key step.
struct ScaleLook {
  const uint8_t *v_scale;
  uint8_t *redo;
  int *any_redo;
  int warps_log2, ctas;
  int *found;  // [kCacheCtas][8], where a sequence and key head has CTAs: what they have found, how many have; zero between launches
};
__device__ __forceinline__ void look_at_scales(const CacheIndex &ix, const ScaleLook &p, int Hkv) {
  // Of a group of warps: a step whose scales are too far apart; what E may be, least and most; the least that it is in a step with values; the most in one
  // with values of zero.
  __shared__ int far[32], least[32], most[32], valued[32], raised[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x - 1, ctas = gridDim.x - 1;
  const int warps = 1 << p.warps_log2, groups = 32 >> p.warps_log2, group = warp >> p.warps_log2;
  const long long pairs = (long long)ix.S * Hkv;
  const int part = cta % p.ctas;  // (several CTAs: one round)
  bool any = false;
  for (long long first = (long long)(cta / p.ctas) * groups; first < pairs; first += (long long)ctas * groups) {
    const long long pair = first + group;
    if (threadIdx.x < 32) far[threadIdx.x] = 0, least[threadIdx.x] = valued[threadIdx.x] = 255, most[threadIdx.x] = raised[threadIdx.x] = 0;
    __syncthreads();
    if (pair < pairs) {
      const int s = (int)(pair / Hkv), h = (int)(pair - (long long)s * Hkv);
      const Sequence q = sequence(ix, s);
      const int len = q.n > 0 ? q.len : 0, low = visible(ix, max(q.len - q.n, 0), q.len).low, sinks = min(ix.sink, low);
      int lo_top = 255, hi_top = 0, valued_top = 255, zero_top = 0, span = 0;
      // the sinks' steps, then those of the window
      const int first_step = max(low / kKeyStep, (sinks + kKeyStep - 1) / kKeyStep), sink_steps = (sinks + kKeyStep - 1) / kKeyStep;
      const int steps = sink_steps + max((len + kKeyStep - 1) / kKeyStep - first_step, 0);
#pragma unroll 2
      for (int i = (part * warps + (warp & (warps - 1))) * 4 + (lane >> 3); i < ((steps + 3) & ~3); i += p.ctas * warps * 4) {
        const int k0 = (i < sink_steps ? i : first_step + i - sink_steps) * kKeyStep + (lane & 7) * 16;
        uint4 b = make_uint4(0u, 0u, 0u, 0u);
        const bool there = i < steps && k0 < len;
        if (there) {
          const int page = page_entry(ix, s, k0);  // (out of range: values of zero, and reported by the tile kernel)
          if ((unsigned)page < (unsigned)ix.n_pages)
            b = __ldcg(reinterpret_cast<const uint4 *>(p.v_scale + ((((size_t)page * Hkv + h) << ix.page_log2) + (k0 & ((1 << ix.page_log2) - 1)))));
        }
        // all 16 bytes, in 16-bit halves; one by one where some token is not seen or a byte has a meaning of its own
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
        uint32_t lows = 0xffffffffu, tops = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t even = w[j] & 0x00ff00ffu, odd = w[j] >> 8 & 0x00ff00ffu;
          lows = __vminu2(lows, __vminu2(even, odd));
          tops = __vmaxu2(tops, __vmaxu2(even, odd));
        }
        int lowest = min(lows & 0xffffu, lows >> 16), highest = max(tops & 0xffffu, tops >> 16), seen = 1, zero = 0;
        if (!there || k0 + 16 > len || (k0 < low && k0 + 16 > sinks) || lowest <= kNoValue || highest == 255) {
          lowest = 255, highest = seen = 0;
#pragma unroll 1
          for (int k = k0; there && k < k0 + 16; ++k) {
            const int i = k - k0, byte = (int)((i < 8 ? i < 4 ? b.x : b.y : i < 12 ? b.z : b.w) >> (8 * (i & 3)) & 255u);
            if (k >= len || (k < low && k >= sinks)) continue;
            seen = 1;
            if (byte <= kNoValue) zero = 1;
            else if (byte < 255) lowest = min(lowest, byte), highest = max(highest, byte);
          }
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
          lowest = min(lowest, __shfl_xor_sync(0xffffffffu, lowest, o));
          highest = max(highest, __shfl_xor_sync(0xffffffffu, highest, o));
          seen |= __shfl_xor_sync(0xffffffffu, seen, o);
          zero |= __shfl_xor_sync(0xffffffffu, zero, o);
        }
        span = max(span, highest - lowest);
        if (seen) {
          // (a tile may see less of the step, and with values of zero among that nothing else)
          const int top = highest > 0 ? highest : kNoValueAs;
          lo_top = min(lo_top, zero ? min(top, kNoValueAs) : top);
          hi_top = max(hi_top, zero ? max(top, kNoValueAs) : top);
          if (highest > 0) valued_top = min(valued_top, top);
          if (zero) zero_top = max(zero_top, max(top, kNoValueAs));
        }
      }
      lo_top = __reduce_min_sync(0xffffffffu, lo_top);
      valued_top = __reduce_min_sync(0xffffffffu, valued_top);
      hi_top = __reduce_max_sync(0xffffffffu, hi_top);
      zero_top = __reduce_max_sync(0xffffffffu, zero_top);
      span = __reduce_max_sync(0xffffffffu, span);
      if (lane == 0) {
        if (span > kScaleSpan) far[group] = 1;
        atomicMin(&least[group], lo_top);
        atomicMin(&valued[group], valued_top);
        atomicMax(&most[group], hi_top);
        atomicMax(&raised[group], zero_top);
      }
    }
    __syncthreads();
    if (pair < pairs && (warp & (warps - 1)) == 0 && lane == 0) {
      int found[5] = {far[group], 255 - least[group], most[group], 255 - valued[group], raised[group]};
      bool all = true;
      if (p.ctas > 1) {
        int *const at = p.found + 8 * (int)pair;
        for (int k = 0; k < 5; ++k) atomicMax(&at[k], found[k]);
        __threadfence();
        all = atomicAdd(&at[5], 1) == p.ctas - 1;
        if (all) {
          __threadfence();
          for (int k = 0; k < 5; ++k) found[k] = atomicExch(&at[k], 0);
          at[5] = 0;
        }
      }
      if (all) {
        const bool redo = found[0] != 0 || found[2] + found[1] - 255 > kScaleRange || found[4] + found[3] - 255 > kScaleSpan;
        p.redo[pair] = redo;
        any |= redo;
      }
    }
    __syncthreads();
  }
  any = __syncthreads_or(any);
  if (threadIdx.x == 0) p.any_redo[cta] = any;
}

constexpr int kSmallPlan = 4096;
// The tiles of a head, sequence by sequence, and the key steps before each.  One CTA; the others look at an e4m3 cache's scales.
template <bool Look>
__global__ void __launch_bounds__(1024) cache_plan_kernel(const CacheIndex ix, int tokens_per_tile, Tile *__restrict__ tiles,
                                                          long long *__restrict__ first, int *__restrict__ head, long long *__restrict__ cuts,
                                                          int32_t *__restrict__ arrivals, int most, int Hkv, bool weigh, const ScaleLook look) {
  __shared__ long long sums[32];
  __shared__ int base[1024];
  __shared__ int costs[kSmallPlan];  // of the first tiles: as a rule all
  __shared__ Sequence own[32];
  auto cost_of = [&](int i) { return i < kSmallPlan ? costs[i] : tiles[i].steps + tiles[i].extra; };
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  pdl_wait();
  // (No word to the tile kernel from those that look: its CTAs come when they have ended, and so to all SMs in their order.  Prompts of 6 x 24 heads took 162 us when they
  // came to the SMs that were free first.)
  if (Look && blockIdx.x > 0) return look_at_scales(ix, look, Hkv);
  pdl_launch_dependents();
  for (int i = t; i < kCacheCtas; i += 1024) arrivals[i] = 0;
  auto upto_lane = [&](long long x) {  // inclusive, over the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    return x;
  };
  auto scan = [&](long long mine, long long &all) {  // exclusive, over the CTA
    const long long x = upto_lane(mine);
    __syncthreads();
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    const long long warps = upto_lane(sums[lane]), before = __shfl_sync(0xffffffffu, warps, max(warp - 1, 0));
    all = __shfl_sync(0xffffffffu, warps, 31);
    return x - mine + (warp > 0 ? before : 0);
  };
  auto largest = [&](long long x) {  // over the CTA
#pragma unroll
    for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
    __syncthreads();
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    x = sums[lane];
#pragma unroll
    for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
  };
  int n_tiles = 0, longest = 1;
  auto make_tile = [&](int i, int s, const Sequence &q, int k) {
    Tile x;
    x.s = s;
    x.row = q.row + k * tokens_per_tile;
    x.tokens = min(tokens_per_tile, q.n - k * tokens_per_tile);
    x.p0 = q.len - q.n + k * tokens_per_tile;
    x.len = q.len;
    const Span<> sp = span_of(ix, x.p0, x.p0 + x.tokens - 1, q.len);
    x.sinks = sp.sinks;
    x.first = sp.first;
    x.steps = sp.steps;
    const Visible v0 = visible(ix, max(x.p0, 0), q.len), v1 = visible(ix, x.p0 + x.tokens - 1, q.len);
    x.every_low = v1.low;
    x.every_end = x.p0 >= 0 ? v0.end : 0;
    x.some_low = v0.low;
    x.some_end = v1.end;
    const int whole = max(x.every_end / kKeyStep - max((x.every_low + kKeyStep - 1) / kKeyStep, x.first), 0) + min(min(ix.sink, x.every_end) / kKeyStep, x.sinks);
    x.extra = weigh ? kTileCost + kMaskCost * max(x.steps - whole, 0) : 0;
    tiles[i] = x;
    const int cost = x.steps + x.extra;
    if (i < kSmallPlan) costs[i] = cost;
    return cost;
  };
  long long before = 0;
  if (ix.S <= 32) {  // a lane a sequence, then a thread a tile
    const Sequence q = lane < ix.S ? sequence(ix, lane) : Sequence{0, 0, 0};
    const int mine = (q.n + tokens_per_tile - 1) / tokens_per_tile;
    const long long upto = upto_lane(mine);
    n_tiles = (int)min(__shfl_sync(0xffffffffu, upto, 31), (long long)most);
    if (warp == 0) {
      base[lane] = (int)min(upto - mine, (long long)most);
      own[lane] = q;
    }
    __syncthreads();
    for (int t0 = 0; t0 < n_tiles; t0 += 1024) {
      const int i = t0 + t;
      int here = 0;
      if (i < n_tiles) {
        int s = 0;  // the last sequence whose tiles begin at i or before
#pragma unroll
        for (int o = 16; o; o >>= 1)
          if (s + o < ix.S && base[s + o] <= i) s += o;
        here = make_tile(i, s, own[s], i - base[s]);
      }
      longest = max(longest, here);
      long long all;
      const long long at = before + scan(here, all);
      if (i < n_tiles) first[i] = at;
      before += all;
    }
  } else {
    for (int s0 = 0; s0 < ix.S; s0 += 1024) {
      const Sequence q = s0 + t < ix.S ? sequence(ix, s0 + t) : Sequence{0, 0, 0};
      const int mine = (q.n + tokens_per_tile - 1) / tokens_per_tile;
      long long all;
      base[t] = (int)min(n_tiles + scan(mine, all), (long long)most);
      __syncthreads();
      for (int i = warp; i < 1024 && s0 + i < ix.S; i += 32) {  // a warp a sequence
        const Sequence q = sequence(ix, s0 + i);
        for (int k = lane; k * tokens_per_tile < q.n && base[i] + k < most; k += 32) make_tile(base[i] + k, s0 + i, q, k);
      }
      n_tiles = (int)min(n_tiles + all, (long long)most);  // (more: starts that do not ascend, which are reported)
      __syncthreads();
    }
    for (int t0 = 0; t0 < n_tiles; t0 += 1024) {
      const int here = t0 + t < n_tiles ? cost_of(t0 + t) : 0;
      longest = max(longest, here);
      long long all;
      const long long at = before + scan(here, all);
      if (t0 + t < n_tiles) first[t0 + t] = at;
      before += all;
    }
  }
  longest = (int)largest(longest);
  const long long per_head = before, total = per_head * Hkv, all_tiles = (long long)n_tiles * Hkv;
  int rounds = (int)max(all_tiles / kCacheCtas - 1, 0LL);
  long long dealt = 0, most_dealt = 0;  // to CTA t, to the one with most
  while (rounds > 0) {
    dealt = 0;
    if (t < kCacheCtas)
      for (int k = 0, i = t % n_tiles, by = kCacheCtas % n_tiles; k < rounds; ++k) {
        dealt += cost_of(i);
        i = i + by < n_tiles ? i + by : i + by - n_tiles;
      }
    most_dealt = largest(dealt);
    if (most_dealt * kCacheCtas <= total) break;
    rounds = min(rounds - 1, (int)(rounds * (total / kCacheCtas) / most_dealt));  // (tiles of very different lengths: fewer of them are dealt)
  }
  if (t == 0) {
    head[0] = n_tiles;
    head[1] = rounds;
    *reinterpret_cast<long long *>(&head[2]) = per_head;
  }
  if (rounds == 0) {  // equal shares, of tiles in not too many parts
    const long long share = max((total + kCacheCtas - 1) / kCacheCtas, (long long)(longest + kMaxParts - 1) / kMaxParts);
    if (t <= kCacheCtas) cuts[t] = min(t * share, total);
    return;
  }
  // the least sum to which shares of at least one step can bring all: every warp looks for it by itself, a lane five CTAs
  __shared__ long long of_cta[kCacheCtas];
  if (t < kCacheCtas) of_cta[t] = dealt;
  long long all;
  scan(dealt, all);
  const long long rest = total - all;  // a tile's step a CTA at least
  long long five[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) five[i] = i * 32 + lane < kCacheCtas ? of_cta[i * 32 + lane] : 1LL << 62;
  // the sum lies in (lo, hi]
  long long lo = (total + kCacheCtas - 1) / kCacheCtas - 1, hi = most_dealt + (rest + kCacheCtas - 1) / kCacheCtas;
  while (hi - lo > 1) {
    const long long sum = (lo + hi) / 2;
    long long shares = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i)
      if (i * 32 + lane < kCacheCtas) shares += max(sum - five[i], 1LL);
#pragma unroll
    for (int o = 16; o; o >>= 1) shares += __shfl_xor_sync(0xffffffffu, shares, o);
    (shares >= rest ? hi : lo) = sum;
  }
  const long long at = scan(t < kCacheCtas ? max(hi - dealt, 1LL) : 0, all);
  if (t <= kCacheCtas) cuts[t] = min(at, rest);
}

// ---------------------------------------------------------------------- attention
template <bool E4m3>
__global__ void __launch_bounds__(Layout<E4m3>::kThreads, 1)
    cache_tile_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const TileParams p) {
  using L = Layout<E4m3>;
  extern __shared__ __align__(1024) unsigned char smem[];
  TileShared &sh = *reinterpret_cast<TileShared *>(smem + L::kOffShared);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const CacheIndex &ix = p.ix;
  volatile int *abort = &sh.abort;

  // ------------------------------------------------------------------ set-up
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1);
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.q_ready[i], 4);
      mbar_init(&sh.v_ready[i], E4m3 ? 4 : 1);
      mbar_init(&sh.codes_free[i], 4);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], 4);
      mbar_init(&sh.p_full[i], 4);
      mbar_init(&sh.pv_done[i], 1);
      for (int q = 0; q < 4; ++q) mbar_init(&sh.m_ready[i][q], 1);
      mbar_init(&sh.o_full[i], 1);
      mbar_init(&sh.out_done[i], 4);
      mbar_init(&sh.drain[i], 1);
      mbar_init(&sh.stored[i], 4);
      mbar_init(&sh.told[i], 1);
    }
    for (int i = 0; i < kPartRing; ++i) {
      mbar_init(&sh.part_full[i], 1);
      mbar_init(&sh.part_empty[i], L::kReaders);
    }
    mbar_init(&sh.o_free, 4);
    for (int i = 0; i < kSteps; ++i) mbar_init(&sh.step_full[i], 1);
    for (int i = 0; i < 8; ++i) mbar_init(&sh.scales_full[i], 1);
    sh.abort = 0;
    for (int i = 0; i < 8; ++i) reinterpret_cast<uint4 *>(sh.zeros)[i] = make_uint4(0u, 0u, 0u, 0u);
    mbar_fence_init();
  }
  if (warp == kWarpQK) {
    tmem_alloc(&sh.tmem_base, 512);
    tmem_relinquish();
  }
  if (warp == kWarpK && lane == 0) {
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  pdl_wait();
  pdl_launch_dependents();
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
  // The announced part n into registers' reach; false: none left (or abort).
  auto part_at = [&](int n) -> const Part * {
    if (!wait(&sh.part_full[n % kPartRing], (n / kPartRing) & 1)) return nullptr;
    return &sh.part[n % kPartRing];
  };
  auto done_with_part = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_empty[n % kPartRing]);
  };
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
  const int page_log2 = ix.page_log2, n_boxes = 128 >> page_log2;
  auto load_pages = [&](unsigned char *dst, const CUtensorMap *map, uint64_t *bar, int h, int page) {
    if (lane == 0) mbar_expect_tx(bar, L::kKey);
    __syncwarp();
    if (lane < n_boxes) {
      unsigned char *to = dst + (lane << (page_log2 + 7));
      tma_load_5d(to, map, bar, 0, 0, 0, h, page);
      if (!E4m3 && n_boxes > 1) tma_load_5d(to + kTileBytes / 2, map, bar, 0, 0, 1, h, page);
    }
  };
  // ------------------------------------------------------------------ roles
  if (warp >= kWarpConvert) {
    setmaxnreg_dec<L::kRegsConvert>();
  } else if (warp >= kWarpQK) {
    setmaxnreg_dec<L::kRegsHelper>();
  }
  if (warp == kWarpK) {
    // ===== the CTA's parts; K and Q producer.  What a step's other warps need to know is said before its copy is waited for.  (Little code: it
    // is one of many places that the warps of an SM are in, see attn_tc.cu.  A warp of its own that looked ahead by five steps, with ten times
    // the instructions, ran at three quarters of the rate.)
    const int n_tiles = __ldcg(&p.head[0]), rounds = __ldcg(&p.head[1]);
    const long long per_head = __ldcg(reinterpret_cast<const long long *>(&p.head[2]));
    const long long u0 = __ldcg(&p.cuts[blockIdx.x]), u1 = __ldcg(&p.cuts[blockIdx.x + 1]);
    const long long dealt = (long long)rounds * gridDim.x;  // tiles
    long long u = u0;  // of the share: the part's first step
    int h, tile, off = 0;  // ... and what of its tile lies before it
    auto share_begins = [&]() {
      // the line's first step, as a step of all heads
      const int h0 = (int)(dealt / n_tiles);
      const int t0 = (int)(dealt - (long long)h0 * n_tiles);
      const long long at = u + h0 * per_head + (t0 > 0 ? __ldcg(&p.first[t0]) : 0);
      h = (int)(at / per_head);
      const long long rest = at - h * per_head;
      tile = 0;
      int hi = n_tiles;  // first[tile] <= rest < first[hi]
      long long begins = 0;
      while (hi - tile > 1) {
        const int step = (hi - tile + 31) / 32, i = tile + lane * step;
        const long long f = i < hi ? __ldcg(&p.first[i]) : 0;
        const int n = __popc(__ballot_sync(0xffffffffu, i < hi && (lane == 0 || f <= rest)));
        begins = __shfl_sync(0xffffffffu, f, n - 1);
        tile += (n - 1) * step;
        hi = min(hi, tile + step);
      }
      off = (int)(rest - begins);
    };
    auto holders = [&](long long at, long long to, int &c0, int &c1) {  // the CTAs whose shares have these steps
      uint32_t n = 0;
#pragma unroll
      for (int c = 0; c < kCacheCtas; c += 32) {
        const long long cut = c + lane < kCacheCtas ? __ldcg(&p.cuts[c + lane]) : 1LL << 62;
        n += (cut <= at ? 1u : 0u) + (cut <= to ? 1u << 16 : 0u);
      }
      n = __reduce_add_sync(0xffffffffu, n);
      c0 = (int)(n & 0xffffu) - 1;
      c1 = (int)(n >> 16) - 1;
    };
    int k = 0;  // tiles of this CTA that it has been dealt so far
    auto next_dealt = [&]() {
      const long long i = blockIdx.x + (long long)k * gridDim.x;
      h = (int)(i / n_tiles);
      tile = (int)(i - (long long)h * n_tiles);
    };
    int g = 0, n = 0;
    auto fetch = [&](int i) {  // lane i: a word of a tile
      return lane < kTileWords ? __ldcg(reinterpret_cast<const int *>(&p.tiles[i]) + lane) : 0;
    };
    h = tile = 0;
    if (rounds > 0) next_dealt();
    else if (u < u1) share_begins();
    int word = rounds > 0 || u < u1 ? fetch(tile) : 0;
    // from a step's first key to that of the lane's box
    const uint32_t ahead = lane < n_boxes ? lane << page_log2 : 0x7fffffff;
    auto key_at = [&](const Tile &t, int i) { return (i < t.sinks ? i : t.first + i - t.sinks) * kKeyStep; };
    auto entry_of = [&](const Tile &t, int k0) {
      return k0 + ahead < (uint32_t)t.len ? __ldcg(ix.table + ((size_t)t.s * ix.table_stride + lane + (k0 >> page_log2))) : ix.n_pages;
    };
    // Announces part m (or the end), and asks for its first pages and the tile behind it.
    bool any;
    int entry = 0;
    auto announce = [&](int m) {
      if (m >= kPartRing && !wait(&sh.part_empty[m % kPartRing], (m / kPartRing - 1) & 1)) return;
      Part &x = sh.part[m % kPartRing];
      const bool from_line = k >= rounds;
      any = !from_line || u < u1;
      if (lane < kTileWords) reinterpret_cast<int *>(&x.t)[lane] = word;
      __syncwarp();
      // (a tile in the line: its extra cost, its steps)
      const int steps = x.t.steps, extra = x.t.extra, a = max(off - extra, 0);
      int b = any ? from_line ? (int)min((long long)steps, off + (u1 - u) - extra) : steps : -1;
      if (b <= a) b = -1, any = false;  // (the share ends before the tile's first step)
      int c0 = blockIdx.x, parts = 1;
      if (any && b - a < steps) {
        int c1;
        holders(u - off + extra, u - off + extra + steps - 1, c0, c1);
        parts = c1 - c0 + 1;
      }
      if (lane == 0) {
        x.h = h;
        x.a = a;
        x.b = b;
        x.c0 = c0;
        x.parts = parts;
        mbar_arrive(&sh.part_full[m % kPartRing]);
      }
      __syncwarp();  // (no other warp writes the ring: this one goes on reading the part)
      if (!any) return;
      entry = entry_of(x.t, key_at(x.t, a));
      if (!from_line) {
        if (++k < rounds) next_dealt();
        else if (u < u1) share_begins();
      } else {
        u += extra + b - off;
        off = 0;
        if (++tile == n_tiles) tile = 0, ++h;
      }
      if (k < rounds || u < u1) word = fetch(tile);
    };
    announce(0);
#pragma unroll 1
    for (; ok && any; ++n) {
      const Part &x = sh.part[n % kPartRing];
      const int a_now = x.a, b = x.b, h_now = x.h;
      const uint32_t len = x.t.len;
      const int sinks = x.t.sinks, shift = x.t.first - x.t.sinks, sink = ix.sink, every_low = x.t.every_low, every_end = x.t.every_end;
      const int32_t *table = ix.table + (size_t)x.t.s * ix.table_stride + lane;
      int k0 = key_at(x.t, a_now);
#pragma unroll 1
      for (int i = a_now; i < b; ++i, ++g) {
        Step &y = sh.step[g % kSteps];
        int page = entry;
        // (out of range: zeros)
        if ((unsigned)page >= (unsigned)ix.n_pages) page = k0 + ahead < len ? checked_page(ix, page) : ix.n_pages;
        if (lane < 8) y.page[lane] = page;
        if (lane == 0) {
          y.key = k0;
          y.h = h_now;
          y.flags = k0 + kKeyStep <= every_end && (k0 >= every_low || k0 + kKeyStep <= sink) ? 0 : kStepMasked;
          if (E4m3) y.seen = 0;
          if (E4m3 && y.flags != 0) {
            const int low = x.t.some_low - k0, end = x.t.some_end - k0;
            if (low > 0 || end < kKeyStep) y.seen = (int)(kStepUnseen | min(max(low, 0), kKeyStep) << 8 | min(max(end, 0), kKeyStep));
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.step_full[g % kSteps]);
        if (i + 1 < b) {
          k0 = (i + 1 < sinks ? i + 1 : i + 1 + shift) * kKeyStep;
          entry = k0 + ahead < len ? __ldcg(table + (k0 >> page_log2)) : ix.n_pages;
        }
        if (g >= 2 && !wait(&sh.s_full[g & 1], ((g - 2) >> 1) & 1)) break;
        load_pages(smem + L::kOffK + (g & 1) * L::kKey, &map_k, &sh.k_full[g & 1], h_now, page);
        if (i == a_now) {
          if (n >= 2 && !wait(&sh.out_done[n & 1], ((n - 2) >> 1) & 1)) {
            ++g;
            break;
          }
          if (lane == 0) {
            unsigned char *q = smem + L::kOffQ + (n & 1) * kTileBytes;
            mbar_expect_tx(&sh.q_full[n & 1], 2 * (128 / p.G * p.G) * 128);
            tma_load_5d(q, &map_q, &sh.q_full[n & 1], 0, 0, x.t.row, 0, h_now);
            tma_load_5d(q + kTileBytes / 2, &map_q, &sh.q_full[n & 1], 0, 0, x.t.row, 1, h_now);
          }
        }
      }
      if (ok) announce(n + 1);  // (before the copies of the last steps are used)
    }
    if (E4m3 && ok) {  // for those who look ahead
      if (lane == 0) {
        sh.step[g % kSteps].flags = kStepEnd;
        mbar_arrive(&sh.step_full[g % kSteps]);
      }
    }
    if (*abort) {
      settle_pair(sh.k_full, g);
      settle_pair(sh.q_full, n + 1);
    }
  } else if (warp == kWarpV) {
    // ===== V producer; e4m3: the scales of a step's tokens too, told of two steps ahead, asked for three
    int g = 0, asked = 0;
    bool ended = !E4m3;
    uint32_t kb = 0, vb = 0;  // scale bytes of keys 4 * lane .. 4 * lane + 3; where there are none, 127 and nothing
    auto ask = [&]() {
      if (ended || !wait(&sh.step_full[asked % kSteps], (asked / kSteps) & 1)) return;
      const Step &y = sh.step[asked % kSteps];
      if (y.flags & kStepEnd) {
        ended = true;
        return;
      }
      const int page = y.page[(lane * 4) >> page_log2];
      kb = 0x7f7f7f7fu, vb = 0u;
      if (page < ix.n_pages) {
        const size_t from = (((size_t)page * p.Hkv + y.h) << page_log2) + ((y.key + lane * 4) & ((1 << page_log2) - 1));
        kb = __ldcg(reinterpret_cast<const uint32_t *>(p.k_scale + from));
        vb = __ldcg(reinterpret_cast<const uint32_t *>(p.v_scale + from));
      }
    };
    auto tell = [&]() {
      if (ended || !ok) return;
      const Step &y = sh.step[asked % kSteps];
      // (bytes with a meaning of their own, and a step with keys that no row sees, come seldom)
      const bool special = (__vcmpeq4(kb, 0xffffffffu) | __vcmpeq4(vb, 0xffffffffu) | __vcmpeq4(kb, 0u)) != 0u || y.seen < 0;
      uint32_t bad = 0u;
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(__byte_perm(kb, 0, 0x0444 | j << 12) >> 1);  // 2^(byte - 127)
      if (__any_sync(0xffffffffu, special)) {
        const int low = y.seen < 0 ? y.seen >> 8 & 255 : 0, end = y.seen < 0 ? y.seen & 255 : kKeyStep;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t k = (kb >> (8 * j)) & 255u, v = (vb >> (8 * j)) & 255u;
          const int i = lane * 4 + j;
          const bool seen = i < end && (i >= low || y.key + i < ix.sink);
          f[j] = k == 255u ? 1.f : cache_scale(k);  // (more than 0: hidden scores of -inf stay -inf)
          if (k == 255u || v == 255u) bad |= 1u << j;
          if (v == 255u || !seen) vb &= ~(255u << (8 * j));  // (nothing)
        }
        bad <<= 4 * (lane & 7);  // a bit a key: eight lanes a word
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, o);
      }
      const uint32_t two = __vmaxu4(vb, vb >> 16), top = __reduce_max_sync(0xffffffffu, max(two & 255u, (two >> 8) & 255u));
      *reinterpret_cast<float4 *>(&sh.k_scale[asked & 7][lane * 4]) = make_float4(f[0], f[1], f[2], f[3]);
      *reinterpret_cast<uint32_t *>(&sh.v_scale[asked & 7][lane * 4]) = vb;
      if ((lane & 7) == 0) sh.bad[asked & 7][lane >> 3] = bad;
      if (lane == 0) sh.top[asked & 7] = top > kNoValue ? (int)top : kNoValueAs;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.scales_full[asked & 7]);
      ++asked;
    };
    for (int i = 0; i < 2; ++i) {
      ask();
      tell();
    }
    ask();
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr || x->b < 0) break;
      const int n_steps = x->b - x->a, every_low = x->t.every_low, every_end = x->t.every_end, some_low = x->t.some_low,
                some_end = x->t.some_end, len = x->t.len, p0 = x->t.p0;
      if (!E4m3) *reinterpret_cast<uint32_t *>(&sh.not_finite[n & 3][lane * 4]) = 0u;
      done_with_part(n);
#pragma unroll 1
      for (int i = 0; i < n_steps; ++i, ++g) {
        const int at = g & 1;
        if (!E4m3 && !wait(&sh.step_full[g % kSteps], (g / kSteps) & 1)) break;
        const Step &y = sh.step[g % kSteps];
        const int page = y.page[lane & 7], h = y.h;
        const bool masked = y.flags & kStepMasked;
        if (g >= 2 && !wait(E4m3 ? &sh.codes_free[at] : &sh.pv_done[at], ((g - 2) >> 1) & 1)) break;
#ifdef HEART_TEST_HOOKS
        if (!(p.test_skip && blockIdx.x == 0 && g == 1))
#endif
        load_pages(smem + (E4m3 ? L::kOffCodes : L::kOffV) + at * L::kKey, &map_v, &sh.v_full[at], h, page);
        if (E4m3) {
          tell();  // of step g + 2
          ask();
        }
        if (!E4m3) {
          if (masked) {
            if (!wait(&sh.v_full[at], (g >> 1) & 1)) {
              ++g;
              break;
            }
            // Values that no row sees are taken out as they are, those that some rows see looked at: [2 dim halves][128 keys][8 x 16 bytes],
            // 16 keys at a time, a lane 16 bytes of each half of every fourth.
            const uint32_t v_at = smem_u32(smem + L::kOffV + at * kTileBytes) + lane * 16;
            const int k0 = y.key;
#pragma unroll 1
            for (int c = 0; c < 128; c += 16) {
              const int key = k0 + c, mine = key + (lane >> 3);
              if (key + 16 <= every_end && (key >= every_low || key + 16 <= ix.sink)) continue;
              if (key >= some_end || (key + 16 <= some_low && key >= ix.sink)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sts_u4(v_at + (j & 1) * (kTileBytes / 2) + (c + 4 * (j >> 1)) * 128, make_uint4(0u, 0u, 0u, 0u));
                continue;
              }
              uint4 v[4], w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) v[j] = lds_u4(v_at + (c + 4 * j) * 128), w[j] = lds_u4(v_at + kTileBytes / 2 + (c + 4 * j) * 128);
              uint32_t out = 0u;   // bits j: key 4 * j of this lane is to be taken out, bits 4 + j: though rows see it
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int kj = mine + 4 * j;
                const bool seen = kj < some_end && (kj >= some_low || kj < ix.sink);
                if (!seen) out |= 1u << j;
                else if (add_zero_times(w[j], add_zero_times(v[j], 0u)) != 0u) out |= 17u << j;
              }
              if (__all_sync(0xffffffffu, out == 0u)) continue;
#pragma unroll
              for (int o = 1; o < 8; o <<= 1) out |= __shfl_xor_sync(0xffffffffu, out, o);  // (the eight lanes of a key)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (out >> j & 1u) {
                  sts_u4(v_at + (c + 4 * j) * 128, make_uint4(0u, 0u, 0u, 0u));
                  sts_u4(v_at + kTileBytes / 2 + (c + 4 * j) * 128, make_uint4(0u, 0u, 0u, 0u));
                }
              }
              if (__any_sync(0xffffffffu, out > 15u)) {  // rows that see such a key: 16 rows for each of a key's lanes
#pragma unroll 1
                for (int j = 0; j < 4; ++j)
#pragma unroll 1
                  for (int r = lane & 7; r < 128 && (out >> (4 + j) & 1u); r += 8) {
                    const Visible see = visible(ix, p0 + p.token_of(r), len);
                    const int kj = mine + 4 * j;
                    if (kj < see.end && (kj >= see.low || kj < ix.sink)) sh.not_finite[n & 3][r] = 1;
                  }
              }
            }
            async_proxy_fence();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.v_ready[at]);
        }
      }
    }
    if (*abort) settle_pair(sh.v_full, g);
  } else if (warp == kWarpQK) {
    // ===== issuer of the score products
    const uint64_t q_desc = smem_desc_sw128(smem_u32(smem + L::kOffQ), 16, 1024);
    const uint64_t k_desc = smem_desc_sw128(smem_u32(smem + L::kOffK), 16, 1024);
    const bool leader = elect_one();
    uint32_t g = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr || x->b < 0) break;
      const int n_steps = x->b - x->a;
      done_with_part(n);
      wait(E4m3 ? &sh.q_ready[n & 1] : &sh.q_full[n & 1], (n >> 1) & 1);
      const uint64_t qd = desc_at(q_desc, (n & 1) * (kTileBytes >> 4));
#pragma unroll 1
      for (int i = 0; i < n_steps; ++i, ++g) {  // S_g = Q K_g^T
        const uint32_t b = g & 1;
        if (g >= 2) wait(&sh.s_free[b], ((g - 2) >> 1) & 1);
        if (E4m3) wait(&sh.scales_full[g & 7], (g >> 3) & 1);  // (for the softmax warps)
        if (!wait(&sh.k_full[b], (g >> 1) & 1)) break;
        tc_fence_after();
        if (leader) {
          const uint64_t kd = desc_at(k_desc, b * (L::kKey >> 4));
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            if (E4m3)  // the high parts of the queries, the low parts
              mma_ss_e4m3(tmem + 128 + b * 128, desc_at(qd, (ks >> 2) * 1024 + (ks & 3) * 2), desc_at(kd, (ks & 3) * 2), idesc_e4m3_f32(128, 128), ks > 0 ? 1u : 0u);
            else
              mma_ss(tmem + 128 + b * 128, desc_at(qd, (ks >> 2) * 1024 + (ks & 3) * 2), desc_at(kd, (ks >> 2) * 1024 + (ks & 3) * 2),
                     idesc_bf16_f32(128, 128, false, false), ks > 0 ? 1u : 0u);
          }
          tc_commit(&sh.s_full[b]);
        }
        __syncwarp();
      }
    }
    drain_products(leader, &sh.drain[0]);
  } else if (warp == kWarpPV) {
    // ===== issuer of the value products
    constexpr uint32_t idesc = E4m3 ? idesc_f16_f32(128, 128, false, true) : idesc_bf16_f32(128, 128, false, true);
    const uint64_t v_desc = smem_desc_sw128(smem_u32(smem + L::kOffV), kTileBytes / 2, 1024);
    const bool leader = elect_one();
    uint32_t g = 0;
#pragma unroll 1
    for (int n = 0; ok; ++n) {
      const Part *x = part_at(n);
      if (x == nullptr || x->b < 0) break;
      const int n_steps = x->b - x->a;
      done_with_part(n);
      if (n > 0) wait(&sh.o_free, (n - 1) & 1);
#pragma unroll 1
      for (int i = 0; i < n_steps; ++i, ++g) {  // O (+)= P_g V_g
        const uint32_t b = g & 1;
        wait(E4m3 ? &sh.v_ready[b] : &sh.v_full[b], (g >> 1) & 1);
        if (!E4m3 && (sh.step[g % kSteps].flags & kStepMasked)) wait(&sh.v_ready[b], (g >> 1) & 1);
        if (!wait(&sh.p_full[b], (g >> 1) & 1)) break;
        tc_fence_after();
        if (leader) {
          const uint64_t vd = desc_at(v_desc, b * (kTileBytes >> 4));
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            mma_ts(tmem, tmem + 384 + b * 64 + ks * 8, desc_at(vd, ks * 128), idesc, (i > 0 || ks > 0) ? 1u : 0u);
          if (i == n_steps - 1) tc_commit(&sh.o_full[n & 1]);
          tc_commit(&sh.pv_done[b]);
        }
        __syncwarp();
      }
    }
    drain_products(leader, &sh.drain[1]);
  } else if (warp >= kWarpConvert) {
    // ===== converters (e4m3): a thread a row of Q, a key of V.  (Little besides the conversion itself: asked for here, the scales took 800
    // clocks a step, of 3300.)
    const int r = tid - kWarpConvert * 32;
    uint32_t n = 0;
    // Q: q = 2^k (high + low), codes of both; the row's place in the first half holds the high parts, in the second the low ones.  A row at
    // a time, a lane four dims of it, so that all of it has been read before anything is written.  (40 heads x 4680 over
    // 33k: 2.84 ms; a thread a row, whose loops keep half a row, 3.03; two and eight rows at once 2.91.)
    auto split_queries = [&]() {
      if (!wait(&sh.q_full[n & 1], (n >> 1) & 1)) return;
      const uint32_t at = smem_u32(smem + L::kOffQ + (n & 1) * kTileBytes);
      const uint32_t from = at + (lane >> 4) * (kTileBytes / 2) + (lane & 1) * 8, to = at + (lane & 3) * 4;
#pragma unroll 1
      for (int i = r & ~31; i < (r | 31); i += kRowsAtOnce) {
        uint2 q[kRowsAtOnce];
        uint32_t top[kRowsAtOnce];
#pragma unroll
        for (int j = 0; j < kRowsAtOnce; ++j) q[j] = lds_u2(from + (i + j) * 128 + ((((lane >> 1) ^ (i + j)) & 7) << 4));
#pragma unroll
        for (int j = 0; j < kRowsAtOnce; ++j) {
          const uint32_t two = __vmaxu2(q[j].x & 0x7fff7fffu, q[j].y & 0x7fff7fffu);
          top[j] = __reduce_max_sync(0xffffffffu, max(two & 0xffffu, two >> 16));
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kRowsAtOnce; ++j) {
          float inv;
          const float scale = code_scale(top[j], inv);
          // (at least a normal number: the -inf of what is hidden is to stay that, for queries of zero and a small scale too)
          const float q_scale = p.scale_log2 * scale;
          if (lane == 0) sh.q_scale[n & 1][i + j] = q_scale < 0x1p-126f ? 0x1p-126f : q_scale;
          uint32_t hi[2], lo[2];
          split_codes(q[j].x, inv, hi[0], lo[0]);
          split_codes(q[j].y, inv, hi[1], lo[1]);
          const uint32_t place = to + (i + j) * 128 + ((((lane >> 2) ^ (i + j)) & 7) << 4);
          sts_u1(place, hi[0] | hi[1] << 16);
          sts_u1(place + kTileBytes / 2, lo[0] | lo[1] << 16);
        }
      }
      async_proxy_fence();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_ready[n & 1]);
      ++n;
    };
    int next_start = 0;  // first step of part n
    bool ended = false;
    // (g runs from -1 on: the queries of a part come two steps ahead of its values)
#pragma unroll 1
    for (int g = -1; ok; ++g) {
      if (g >= 0) {
        if (g >= next_start) break;  // (the end: parts are taken ahead)
        const uint32_t b = g & 1;
        const bool v_there = mbar_test_wait(&sh.v_full[b], (g >> 1) & 1), p_there = g < 2 || mbar_test_wait(&sh.pv_done[b], ((g - 2) >> 1) & 1);
        if (!__all_sync(0xffffffffu, v_there && p_there)) {
          if (!wait(&sh.v_full[b], (g >> 1) & 1)) break;
          if (g >= 2 && !wait(&sh.pv_done[b], ((g - 2) >> 1) & 1)) break;
        }
        const uint32_t to = smem_u32(smem + L::kOffV + b * kTileBytes) + r * 128;
        const int vs = sh.v_scale[g & 7][r];
        const float f = vs == 0 ? 0.f : cache_scale(max(vs - sh.top[g & 7] + 127, 1));
        const uint32_t f2 = pack_f16x2(f, f);
        // (Codes behind a sequence's end may be no numbers, and 0 * NaN is NaN.  Masked with four instructions in the loop, 40 heads x 4680 over 33k took
        // 3.48 ms instead of 3.03.)
        const uint32_t from = vs == 0 ? smem_u32(sh.zeros) : smem_u32(smem + L::kOffCodes + b * kCodeBytes) + r * 128;
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {  // 16 dims (fetches of instructions are what is short: unrolled by 1, 2 and 4, 6 prompts x 24 heads 161, 165 and 173 us)
          const uint4 w = lds_u4(from + (((j ^ r) & 7) << 4));
          const uint32_t half = to + (j >> 2) * (kTileBytes / 2);
          sts_u4(half + ((((j & 3) * 2) ^ (r & 7)) << 4), make_uint4(mul_f16x2(codes_to_f16x2(w.x), f2), mul_f16x2(high_codes_to_f16x2(w.x), f2),
                                                                     mul_f16x2(codes_to_f16x2(w.y), f2), mul_f16x2(high_codes_to_f16x2(w.y), f2)));
          sts_u4(half + ((((j & 3) * 2 + 1) ^ (r & 7)) << 4), make_uint4(mul_f16x2(codes_to_f16x2(w.z), f2), mul_f16x2(high_codes_to_f16x2(w.z), f2),
                                                                         mul_f16x2(codes_to_f16x2(w.w), f2), mul_f16x2(high_codes_to_f16x2(w.w), f2)));
        }
        async_proxy_fence();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.v_ready[b]);
          mbar_arrive(&sh.codes_free[b]);
        }
      }
      while (ok && !ended && next_start <= g + 2) {
        const Part *x = part_at(n);
        ended = x == nullptr || x->b < 0;
        if (ended) break;
        next_start += x->b - x->a;
        done_with_part(n);
        split_queries();
      }
    }
  } else {
    // ===== softmax / correction / output: thread = one row
    setmaxnreg_inc<L::kRegsSoftmax>();
    const uint32_t w = warp >> 2, quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t o_addr = tmem + (quarter << 21), s_addr = o_addr + 128, p_addr = o_addr + 384;
    float c = p.scale_log2;
    auto arrive = [&](uint64_t *bar) {  // this warp's tensor-memory accesses so far are ordered before it
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    uint32_t g0 = 0, nt = 0;  // key steps before the present part, parts before it
    int n_steps = 0, h = 0;   // of the present part; this warpgroup's next step of it
    bool leads = w == 0;
    uint32_t pending = 0;     // the part before is this warpgroup's to write: 1 behind its first step of the next one, 2 before
    bool live = true;
    float m_ref = kNoReference, l_run = 0.f;
    int first_top = 0;        // e4m3: the largest scale byte of the part's first step
    enum { kNothing, kNotThere, kMask, kRescale } why = kNothing;  // why the loop over the steps was left
    bool masked = false;
    float alpha = 1.f;
    auto advance = [&]() -> bool {  // steps 0, 3, 5, 7 .. and 1, 2, 4, 6 ..; true if the output of the part before comes first
      const bool first = h < 2;
      h += first ? 3 - 2 * h : 2;
      return first && pending != 0;
    };
    // Hidden keys of step g get a score of -inf; rows that see a key or value that is not finite are marked.
    auto mask_keys = [&](uint32_t g) {
      const uint32_t s_at = s_addr + (g & 1) * 128;
      const Part &x = sh.written[nt & 1][warp];
      const int k0 = sh.step[g % kSteps].key;
      const Visible v = visible(ix, x.t.p0 + p.token_of(row), x.t.len);
      const int end = v.end - k0, low = v.low - k0, sink = ix.sink - k0;
      tc_fence_after();
      auto below = [](int n) { return n <= 0 ? 0u : 0xffffffffu >> (32 - min(n, 32)); };  // bits 0 .. n - 1
#pragma unroll 1
      for (int col = 0; col < 128; col += 32) {
        const uint32_t seen = below(end - col) & (~below(low - col) | below(sink - col));
        if (__all_sync(0xffffffffu, seen == 0xffffffffu)) continue;
        uint32_t y[32];
        tmem_ld32(s_at + col, y);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (!(seen >> i & 1u)) y[i] = 0xff800000u;
        tmem_st32(s_at + col, y);
      }
      tmem_wait_st();
#pragma unroll 1
      for (int j = 0; E4m3 && j < 4; ++j)
#pragma unroll 1
        for (uint32_t todo = sh.bad[g & 7][j]; todo; todo &= todo - 1) {
          const int k = j * 32 + __ffs(todo) - 1;
          if (k < end && (k >= low || k < sink)) l_run = __uint_as_float(0x7fc00000u);
        }
    };
    auto end_part = [&]() {
      if (n_steps == 0) return;
      const int last = n_steps - 1;
      const bool mine = leads == (last == 0 || (last > 2 && (last & 1)));  // had the last step
      leads = !mine;
      const bool at_once = n_steps == 1;
      if (mine == at_once) {
        pending = at_once ? 2 : 1;
        if (at_once) sh.l[nt & 3][w ^ 1][row] = make_float2(0.f, kNoReference);  // (the other one had no step)
      }
      g0 += n_steps;
      ++nt;
    };
    int n_part = 0;
    uint32_t n_stored = 0;  // parts that this warpgroup has left in the workspace
    auto next = [&]() {
      const Part *x = part_at(n_part);
      live = x != nullptr && x->b >= 0;
      if (!live) return;
      if (lane < kPartWords) reinterpret_cast<int *>(&sh.written[nt & 1][warp])[lane] = reinterpret_cast<const int *>(x)[lane];
      n_steps = x->b - x->a;
      done_with_part(n_part);  // (a warp barrier: all lanes see the copy)
      ++n_part;
      h = leads ? 0 : 1;
      m_ref = kNoReference;
      l_run = 0.f;
    };
    for (;;) {
      if (pending != 2)
#pragma unroll 1
      while (h < n_steps) {
        const uint32_t g = g0 + h, b = g & 1, s_at = s_addr + b * 128, p_at = p_addr + b * 64;
        const bool m_there = mbar_try_wait(&sh.m_ready[b ^ 1][quarter], ((g - 1) >> 1) & 1, kShortWait) || g == 0;
        const bool there = mbar_try_wait(&sh.s_full[b], (g >> 1) & 1, kShortWait) && m_there;
        if (__builtin_expect(!__all_sync(0xffffffffu, there), 0)) {
          why = kNotThere;
          break;
        }
        bool special = sh.step[g % kSteps].flags & kStepMasked;
        if (E4m3) {
          const uint4 bad = *reinterpret_cast<const uint4 *>(sh.bad[g & 7]);
          special |= (bad.x | bad.y | bad.z | bad.w) != 0u;
        }
        tc_fence_after();
        float shift = 0.f, l_factor = 1.f;  // e4m3: E of the step, 2^(E of the part's first step - E)
        if (E4m3) {
          c = sh.q_scale[nt & 1][row];
          if (h < 2) first_top = sh.top[g0 & 7];
          const int top = sh.top[g & 7];
          shift = (float)(top - 127);
          l_factor = cache_scale(min(max(first_top - top + 127, 1), 254));
        }
        const float m_prev = h > 0 ? sh.m[b ^ 1][row] : kNoReference;
        uint64_t sums[2] = {0ull, 0ull};
        bool moved = false;
        auto new_reference = [&](float x_max) -> bool {
          const bool grow = x_max > m_ref + (E4m3 ? kMaxGrowthE4m3 : kMaxGrowth);
          const float m_new = grow ? x_max + (E4m3 ? kHeadroomE4m3 : kHeadroom) : m_ref;
          sh.m[b][row] = m_new;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.m_ready[b][quarter]);
          if (__builtin_expect(!__any_sync(0xffffffffu, grow), 1)) return false;
          moved = true;
          alpha = ex2(m_ref - m_new);
          l_run *= alpha;
          m_ref = m_new;
          return true;
        };
        if (__builtin_expect(special && !masked, 0)) {
          why = kMask;
          break;
        }
        uint32_t s[128], pk[32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(s_at + q * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[q * 32]));
        l_run *= ex2(m_ref - m_prev);
        m_ref = m_prev;
        tmem_wait_ld();
        arrive(&sh.s_free[b]);
        if (E4m3) {
#pragma unroll
          for (int i = 0; i < 128; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(&sh.k_scale[g & 7][i]);
            float a0, a1;
            unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), pack_f32x2(f.x, f.y)), a0, a1);
            s[i] = __float_as_uint(a0), s[i + 1] = __float_as_uint(a1);
            unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), pack_f32x2(f.z, f.w)), a0, a1);
            s[i + 2] = __float_as_uint(a0), s[i + 3] = __float_as_uint(a1);
          }
        }
        const uint64_t c2 = pack_f32x2(c, c);
        uint64_t neg_m2;
        bool again = false;
#pragma unroll 1
        do {
          neg_m2 = pack_f32x2(shift - m_ref, shift - m_ref);
          sums[0] = sums[1] = 0ull;
          exp32<E4m3>(&s[0], c2, neg_m2, &pk[0], sums);
          const float x_max = fmaf(fmaxf(max64(&s[0]), max64(&s[64])), c, shift);
          again = !again && new_reference(x_max);
        } while (__builtin_expect(again, 0));
        const bool p_done = g < 2 || mbar_test_wait(&sh.pv_done[b], ((g - 2) >> 1) & 1);
        exp32<E4m3>(&s[32], c2, neg_m2, &pk[16], sums);
        if (__builtin_expect(!__all_sync(0xffffffffu, p_done), 0)) wait(&sh.pv_done[b], ((g - 2) >> 1) & 1);
        tc_fence_after();
        tmem_st32(p_at, pk);
        exp32<E4m3>(&s[64], c2, neg_m2, &pk[0], sums);
        exp32<E4m3>(&s[96], c2, neg_m2, &pk[16], sums);
        tmem_st32(p_at + 32, pk);
        float s0, s1, s2, s3;
        unpack_f32x2(sums[0], s0, s1);
        unpack_f32x2(sums[1], s2, s3);
        l_run = E4m3 ? fmaf((s0 + s1) + (s2 + s3), l_factor, l_run) : l_run + ((s0 + s1) + (s2 + s3));
        if (h >= n_steps - 3) {
          sh.l[nt & 3][w][row] = make_float2(l_run, m_ref);
          if (E4m3) sh.first_top[nt & 3] = first_top;
        }
        if (!ok) break;
        if (__builtin_expect(moved && h > 0, 0)) {
          why = kRescale;
          break;
        }
        tmem_wait_st();
        arrive(&sh.p_full[b]);
        masked = false;
        if (__builtin_expect(advance(), 0)) break;
      }
      if (why != kNothing && ok) {
        const uint32_t g = g0 + h, b = g & 1;
        if (why == kNotThere) {
          if (g > 0) wait(&sh.m_ready[b ^ 1][quarter], ((g - 1) >> 1) & 1);
          wait(&sh.s_full[b], (g >> 1) & 1);
        } else if (why == kMask) {
          mask_keys(g);
          masked = true;
        } else {
          // O changes scale: the products of the steps before have to be complete
          if (wait(&sh.pv_done[b ^ 1], ((g - 1) >> 1) & 1)) {
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
            tmem_wait_st();
            arrive(&sh.p_full[b]);
            masked = false;
            advance();
          }
        }
        const bool whole_step = why == kRescale;
        why = kNothing;
        if (ok && !whole_step) continue;
      }
      if (!ok) break;
      if (pending) {
        // ===== the output of the part before
        const uint32_t w_last = pending == 2 ? w : w ^ 1;
        pending = 0;
        const uint32_t q_buf = (nt - 1) & 1;
        const Part &to = sh.written[q_buf][warp];
        if (!wait(&sh.o_full[q_buf], ((nt - 1) >> 1) & 1)) break;
        tc_fence_after();
        const float2 last = sh.l[(nt - 1) & 3][w_last][row], other = sh.l[(nt - 1) & 3][w_last ^ 1][row];
        float l = last.x + other.x * ex2(other.y - last.y), m = last.y, o_factor = 1.f;
        if (E4m3) {  // O and the row's sum in one unit: m less by E of the first step
          o_factor = cache_scale(sh.first_top[(nt - 1) & 3]);
          m -= (float)(sh.first_top[(nt - 1) & 3] - 127);
        }
        const int n_rows = to.t.tokens * p.G;
        const bool whole = to.a == 0 && to.b == to.t.steps;
        const uint32_t out = smem_u32(smem + L::kOffQ + q_buf * kTileBytes + quarter * (kTileBytes / 4));  // the place of its Q: 32 rows a warp
        const int slot = 2 * blockIdx.x + (to.a == 0 ? 1 : 0);
        // e4m3: a row without any key whose query is not finite has sums that are no numbers
        const bool none = E4m3 && to.t.p0 + p.token_of(row) < 0;
        if (none) l = 0.f;
        if (!E4m3 && sh.not_finite[(nt - 1) & 3][row]) l = __uint_as_float(0x7fc00000u);
        // 64 dims of the row as bf16, O / l, into shared memory
        auto stage = [&](const uint32_t (&v)[64], int half, float inv) {
          const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint32_t x[4];
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
              float a0, a1, a2, a3;
              unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[i * 8 + 2 * k]), __uint_as_float(v[i * 8 + 2 * k + 1])), inv2), a0, a1);
              unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[i * 8 + 2 * k + 2]), __uint_as_float(v[i * 8 + 2 * k + 3])), inv2), a2, a3);
              x[k] = pack_bf16x2(a0, a1);
              x[k + 1] = pack_bf16x2(a2, a3);
            }
            if (none) x[0] = x[1] = x[2] = x[3] = 0u;
            sts_u4(out + half * (kTileBytes / 8) + lane * 128 + ((i ^ (lane & 7)) << 4), make_uint4(x[0], x[1], x[2], x[3]));
          }
        };
        float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          uint32_t v[64];
          tmem_ld32(o_addr + half * 64, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
          tmem_ld32(o_addr + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
          tmem_wait_ld();
          if (half == 1) arrive(&sh.o_free);
          // A code that is no number, in a token that some rows see and others do not, has reached them all (0 * NaN is NaN): rows do it
          // again.  (Looked at by the converters, in the steps that some row does not see whole, 12 x 4680 over 12 680 took 415 us instead of 390.)
          if (E4m3) {
            uint64_t zero = 0ull;
#pragma unroll
            for (int i = 0; i < 64; i += 2) zero = fma_f32x2(pack_f32x2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), 0ull, zero);
            if (zero != 0ull && l == l && !none && row < n_rows) {
              p.redo[(size_t)to.t.s * p.Hkv + to.h] = 1;
              p.any_redo[0] = 1;
            }
          }
          if (whole) {
            stage(v, half, inv * o_factor);
          } else if (row < n_rows) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              __stcg(&p.parts[((size_t)slot * 32 + half * 16 + i) * 128 + row],
                     make_float4(__uint_as_float(v[4 * i]) * o_factor, __uint_as_float(v[4 * i + 1]) * o_factor, __uint_as_float(v[4 * i + 2]) * o_factor,
                                 __uint_as_float(v[4 * i + 3]) * o_factor));
          }
        }
        bool write = whole;
        if (!whole) {
          if (row < n_rows) __stcg(&p.part_l[slot * 128 + row], make_float2(l, m));
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.stored[w]);
          if (quarter == 0) {
            if (!wait(&sh.stored[w], n_stored & 1)) break;
            if (lane == 0) {
              __threadfence();  // (of what the warpgroup has stored, which the barrier has shown this thread)
              sh.last[w] = atomicAdd(&p.arrivals[to.c0], 1) == to.parts - 1;
              __threadfence();
              mbar_arrive(&sh.told[w]);
            }
            __syncwarp();
          }
          if (!wait(&sh.told[w], n_stored & 1)) break;
          ++n_stored;
          write = sh.last[w] != 0;
          if (write && row < n_rows) {
            auto place = [&](int i) { return 2 * (to.c0 + i) + (i == 0 ? 1 : 0); };
            m = kNoReference;
            l = 0.f;
#pragma unroll 4
            for (int i = 0; i < to.parts; ++i) m = fmaxf(m, __ldcg(&p.part_l[place(i) * 128 + row]).y);
#pragma unroll 4
            for (int i = 0; i < to.parts; ++i) {
              const float2 lm = __ldcg(&p.part_l[place(i) * 128 + row]);
              l = fmaf(lm.x, ex2(lm.y - m), l);
            }
            inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              uint32_t v[64];
#pragma unroll
              for (int i = 0; i < 64; ++i) v[i] = 0u;
#pragma unroll 1
              for (int i = 0; i < to.parts; ++i) {
                const float f = ex2(__ldcg(&p.part_l[place(i) * 128 + row]).y - m);
                const float4 *src = &p.parts[((size_t)place(i) * 32 + half * 16) * 128 + row];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                  const float4 y = __ldcg(src + k * 128);
                  v[4 * k] = __float_as_uint(fmaf(y.x, f, __uint_as_float(v[4 * k])));
                  v[4 * k + 1] = __float_as_uint(fmaf(y.y, f, __uint_as_float(v[4 * k + 1])));
                  v[4 * k + 2] = __float_as_uint(fmaf(y.z, f, __uint_as_float(v[4 * k + 2])));
                  v[4 * k + 3] = __float_as_uint(fmaf(y.w, f, __uint_as_float(v[4 * k + 3])));
                }
              }
              stage(v, half, inv);
            }
          }
        }
        if (write) {
          __syncwarp();
          // two rows at a time, 16 lanes each
          uint16_t *o_row = p.O + (long long)to.t.row * p.qt + (long long)(to.h * p.G) * p.qh + (lane & 15) * 8;
#pragma unroll 1
          for (int i = 0; i < 16; ++i) {
            const int mine = i * 2 + (lane >> 4), r = (int)quarter * 32 + mine, piece = lane & 15;
            const uint4 v = lds_u4(out + (piece >> 3) * (kTileBytes / 8) + mine * 128 + (((piece ^ mine) & 7) << 4));
            const int token = p.token_of(r);
            if (r < n_rows) *reinterpret_cast<uint4 *>(o_row + (long long)token * p.qt + (long long)(r - token * p.G) * p.qh) = v;
          }
          if (p.lse != nullptr && row < n_rows)
            p.lse[(long long)(to.t.row + p.token_of(row)) * p.Hq + to.h * p.G + row - p.token_of(row) * p.G] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
        async_proxy_fence();  // (copies come to the place of Q)
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.out_done[q_buf]);
      }
      if (h < n_steps) continue;
      if (!live) break;
      end_part();
      next();
    }
  }

  // ------------------------------------------------------------------ tear-down
  tc_fence_before();
  __syncthreads();
  if (warp == kWarpQK) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (tid == 0 && sh.abort) atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
}

template <bool E4m3>
cudaError_t launch(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const TileParams &p, cudaStream_t s) {
  cudaError_t e = allow_shared_memory(cache_tile_kernel<E4m3>, kSmem<E4m3>);
  if (e != cudaSuccess) return e;
  return launch_pdl(cache_tile_kernel<E4m3>, dim3(kCacheCtas), dim3(Layout<E4m3>::kThreads), kSmem<E4m3>, s, mq, mk, mv, p);
}

}  // namespace

cudaError_t launch_cache_tiles(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                               void *O, float *lse, cudaStream_t s, int *launches) {
  CUtensorMap mq, mk, mv;
  const int halves = g.page == 128 ? 2 : 1;
  if (!make_query_map(&mq, Q, g) || !make_pool_map(&mk, c.k, g, g.page, halves) || !make_pool_map(&mv, c.v, g, g.page, halves)) return cudaErrorInvalidValue;
  TileParams p = {};
  p.ix = ix;
  p.tiles = reinterpret_cast<const Tile *>(w.tiles);
  p.first = w.tile_first;
  p.head = w.tile_head;
  p.cuts = w.cuts;
  p.arrivals = w.arrivals + kCacheCtas;
  p.parts = reinterpret_cast<float4 *>(w.parts);
  p.part_l = w.part_l;
  p.O = static_cast<uint16_t *>(O);
  p.lse = lse;
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.qt = g.qt;
  p.qh = g.qh;
  p.Hq = g.Hq;
  p.Hkv = g.Hkv;
  p.G = g.G;
  p.inv_G = (65536u + g.G - 1) / g.G;
  p.test_skip = g.test_skip;
  p.scale_log2 = (float)(g.scale * 1.4426950408889634);
  p.redo = w.redo;
  p.any_redo = w.any_redo;
  const int most = (int)cache_max_tiles(g);
  const bool weigh = (long long)most * g.Hkv >= 2 * kCacheCtas;
  cudaError_t e;
  int looked = 0;
  if (g.e4m3) {  // CTAs that look at scales: as many warps a sequence and key head as leave one for each, or a CTA for every 16384 tokens that it may have (one: a
                 // prompt of 512, 12 heads, 28 us; twelve: 31; 100 tokens of one head over 200k: 185 with one, 177 with thirteen)
    ScaleLook look = {c.v_scale, w.redo, w.any_redo, 5, 1, w.found};
    const long long pairs = (long long)g.S * g.Hkv;
    while (look.warps_log2 > 0 && pairs > (long long)(kCacheCtas - 1) << (5 - look.warps_log2)) --look.warps_log2;
    const int groups = 32 >> look.warps_log2;
    const long long rounds = ((long long)g.table_stride * g.page + 16383) / 16384;
    look.ctas = (int)std::max(std::min((kCacheCtas - 1) / pairs, rounds), 1LL);
    looked = (int)std::min((pairs + groups - 1) / groups * look.ctas, (long long)kCacheCtas - 1);
    e = launch_pdl(cache_plan_kernel<true>, dim3(1 + looked), dim3(1024), 0, s, ix, 128 / g.G, reinterpret_cast<Tile *>(w.tiles), w.tile_first, w.tile_head,
                   w.cuts, p.arrivals, most, g.Hkv, weigh, look);
  } else {
    e = launch_pdl(cache_plan_kernel<false>, dim3(1), dim3(1024), 0, s, ix, 128 / g.G, reinterpret_cast<Tile *>(w.tiles), w.tile_first, w.tile_head, w.cuts,
                   p.arrivals, most, g.Hkv, weigh, ScaleLook{});
  }
  if (e != cudaSuccess) return e;
  ++*launches;
  e = g.e4m3 ? launch<true>(mq, mk, mv, p, s) : launch<false>(mq, mk, mv, p, s);
  if (e != cudaSuccess) return e;
  ++*launches;
  return g.e4m3 ? launch_cache_redo(g, ix, w, Q, c, O, lse, looked, s, launches) : cudaSuccess;
}

}  // namespace heart
