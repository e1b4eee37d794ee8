// Cross attention: geometry, workspace, and what its two kernels share.
#pragma once
#include <algorithm>

#include "cache.cuh"

namespace heart {

// Geometry derived from a validated heart_cross_config.
struct CrossGeom {
  int S, T, Tk, Hq, Hkv, G, max_q;
  long long qt, qh, kt, kh;  // element strides: Q and O, K and V
  double scale;
  int test_skip;  // test-hook builds only (see the attention kernels)
};

struct CrossWorkspace {
  int32_t *status;    // [64] word 0: sticky device-check code
  int32_t *arrivals;  // [kCacheCtas] parts of a shared tile that are there (zero between launches)
  float *parts;       // [2 * kCacheCtas][128][128] parts of tiles: unnormalised sums of values
  float2 *part_l;     // [2 * kCacheCtas][128] their row sums and references
  size_t bytes;
};

__host__ inline CrossWorkspace carve_cross(void *base) {
  CrossWorkspace w;
  char *p = static_cast<char *>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char *at = p + off;
    off += align256(bytes);
    return at;
  };
  w.status = reinterpret_cast<int32_t *>(take(64 * sizeof(int32_t)));
  w.arrivals = reinterpret_cast<int32_t *>(take(kCacheCtas * sizeof(int32_t)));
  w.parts = reinterpret_cast<float *>(take(sizeof(float) * 2 * kCacheCtas * 128 * kD));
  w.part_l = reinterpret_cast<float2 *>(take(sizeof(float2) * 2 * kCacheCtas * 128));
  w.bytes = off;
  return w;
}

int make_cross_geom(const heart_cross_config *c, CrossGeom *g);

// Whether all rows are few tiles of 16.  The kernel for few rows takes any number of them, and reads keys and values as often as it has tiles: its smaller share of fixed costs
// is worth that here, as long as the keys are not many.  (16 tiles, 8 heads of 8 x 4 over 500: 7.8 us by tiles of 8 rows, 9.6 of 16, 11.3 by the kernel for tiles of 128; over 2000
// 10.4, 12.0 and 17.5.  24 tiles, 12 heads x 32 over 500: 7.8, 9.5 and 11.5.  36, 12 heads x 48: 9.3, of 128 11.9.)
__host__ inline bool few_rows(const CrossGeom &g) {
  constexpr long long kFewTiles = 24;
  return ((long long)g.T * g.G + 15LL * (g.S < g.T ? g.S : g.T)) / 16 * g.Hkv <= kFewTiles;
}
// Key steps that a CTA has by tiles of `rows` rows: of sequences taken as alike, with Tk / S keys each.
__host__ inline double key_steps(const CrossGeom &g, int rows) {
  const long long sequences = g.S < g.T ? g.S : g.T, each = ((long long)g.T * g.G + sequences - 1) / sequences;
  const double steps = g.Tk / g.S / kKeyStep + 1, tiles = (double)(sequences * ((each + rows - 1) / rows) * g.Hkv);
  return steps * std::max(tiles / kCacheCtas, 1.0 / kMaxParts);
}

// The kernel that a call takes: by 8 or 16 rows, by tiles, by pairs of CTAs.
enum class CrossKernel { kRows8, kRows16, kTiles, kPairs };
__host__ inline CrossKernel cross_kernel(const CrossGeom &g) {
  const long long most_rows = (long long)g.max_q * g.G;  // of a sequence and key head
  if (most_rows <= 8) return CrossKernel::kRows8;
  if (few_rows(g)) {
    // Tiles of 16 rows where a CTA then has this many steps less (a step of 16 rows takes 1.06 us, of 8 rows 0.8, and the launch 3 us more), and tiles of 128 where it would still have
    // many.  8, 16 and 128 rows of one head x 370 over 4000 18.1, 18.2 and 20.9 us, over 8000 25.6, 22.9 and 23.2, over 32 000 69.0, 50.2 and 38.8; 8 heads of 8 x 4 over 8000 20.5, 20.1 and
    // 23.5, over 32 000 56.9, 37.0 and 44.9; 12 heads x 32 over 8000 25.6, 22.7 and 24.6, over 32 000 69.9, 51.7 and 51.2; 24 heads x 16 over 4000 18.2 and 16.1.  (Of 306
    // sizes, over 64 to 150 000, what is chosen takes 1.3 % longer than the best one in the mean, 23 % at most: one head x 370 over 1000, where 8 rows take 14.7 and 16 rows 12.0.)
    constexpr double kStepsSaved = 5, kManySteps = 28;
    const double by16 = key_steps(g, 16);
    if (key_steps(g, 8) - by16 < kStepsSaved) return CrossKernel::kRows8;
    if (by16 <= kManySteps) return CrossKernel::kRows16;
  }
  if (most_rows <= kRowsOfRowsKernel) return CrossKernel::kRows16;
  // Pairs of CTAs, where a sequence may have more rows than a tile, if there are many tiles a CTA or more keys and values than L2 keeps.  (Half of the traffic, and of its power, against
  // an uneven finish: 2 x 40 heads x 32760 over 343 518 us, 537 by single CTAs, and 598 and 614 for most of a second on end; 12 heads x 32760 over 512 111 and 108, x 4680 29 and 23; x 1000 over
  // 32760 182 and 244; 8 x 8 heads x 2000 over 8000 494 and 520.)
  const long long tiles = ((long long)g.T * g.G + 127) / 128 * g.Hkv, keys_bytes = (long long)g.Tk * g.Hkv * 4 * kD;
  const bool pairs = (long long)g.max_q > 128 / g.G && (tiles >= 32 * kCacheCtas || keys_bytes > 64 << 20);
  return pairs ? CrossKernel::kPairs : CrossKernel::kTiles;
}

// ix: row_start and kv_len are the starts of the queries and the numbers of keys, table the first rows of the keys, table_stride the rows of K.
cudaError_t launch_cross_rows(const CrossGeom &g, const CacheIndex &ix, const CrossWorkspace &w, const void *Q, const void *K, const void *V, void *O,
                              float *lse, bool eight, cudaStream_t s, int *launches);
cudaError_t launch_cross_tiles(const CrossGeom &g, const CacheIndex &ix, const CrossWorkspace &w, const void *Q, const void *K, const void *V, void *O,
                               float *lse, bool pair, cudaStream_t s, int *launches);

// K or V as (64 dims, row, dim half, head): a box is one or both halves of `rows` rows of one head, from any row on, 128-byte rows, swizzled.
bool make_states_map(CUtensorMap *m, const void *base, const CrossGeom &g, int rows, int halves);

#ifdef __CUDACC__
struct SequenceWords {
  int r0, r1, len, k0;
};
__device__ __forceinline__ SequenceWords cross_sequence_words(const CacheIndex &ix, int s) {
  return {__ldcg(&ix.row_start[s]), __ldcg(&ix.row_start[s + 1]), __ldcg(&ix.kv_len[s]), __ldcg(&ix.table[s])};
}
// A sequence as its arrays describe it, brought into range (and reported) where they do not hold what they should.
__device__ __forceinline__ Sequence cross_sequence(const CacheIndex &ix, const SequenceWords &w) {
  int r0 = w.r0, r1 = w.r1, len = w.len, k0 = w.k0;
  const int rows = ix.table_stride;
  if (r0 < 0 || r1 < r0 || r1 > ix.T || len < 0 || len > rows || (len > 0 && (k0 < 0 || k0 > rows - len))) {
    atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
    r0 = min(max(r0, 0), ix.T);
    r1 = min(max(r1, r0), ix.T);
    len = min(max(len, 0), rows);
  }
  return {r0, r1 - r0, len, min(max(k0, 0), rows - len)};
}
__device__ __forceinline__ Sequence cross_sequence(const CacheIndex &ix, int s) { return cross_sequence(ix, cross_sequence_words(ix, s)); }
#endif

}  // namespace heart
