// A paged cache of keys and values: geometry, workspace, and the device code that the kernels on it share.
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace heart {

constexpr int kKeyStep = 128;  // keys are processed in steps of 128, from token 0 of a sequence
constexpr int kCacheCtas = 148;  // persistent CTAs of an attention launch, one per SM

// Geometry derived from a validated heart_cache_config.
struct CacheGeom {
  int S, T, Hq, Hkv, G, page, n_pages, table_stride, e4m3, max_new, causal, window, sink;
  long long qt, qh, kvt, kvh;  // element strides: Q and O, packed K and V
  long long pp, ph, pt;        // the pools
  double scale;
  int test_skip;  // test-hook builds only (see the attention kernels)
};

// What the kernels on the cache read on the device.
struct CacheIndex {
  const int32_t *table, *row_start, *kv_len;
  int32_t *status;
  int S, T, page_log2, n_pages, table_stride;
  int causal, window, sink;
};

struct CacheWorkspace {
  int32_t *status;    // [64] word 0: sticky device-check code
  int32_t *arrivals;  // [2][kCacheCtas] parts of a shared tile that are there: the rows kernel's (zero between launches), the tile kernel's
  int *found;         // [kCacheCtas][8] what CTAs that look at the scales of one sequence and key head have found (zero between launches)
  float *parts;       // [2 * kCacheCtas][128][128] parts of tiles: unnormalised sums of values
  float2 *part_l;     // [2 * kCacheCtas][128] their row sums and references
  void *tiles;        // [max_tiles] tiles of a head (see cache_tiles.cu)
  long long *tile_first;  // [max_tiles + 1] cost of the tiles before a tile, in key steps
  int *tile_head;     // [64] number of tiles of a head, rounds of them that are dealt
  long long *cuts;    // [kCacheCtas + 1] the CTAs' shares of the other ones
  int *any_redo;      // [kCacheCtas] 1 where a CTA that looked at the scales found something to do again by rows
  uint8_t *redo;      // [S * Hkv] 1: the sequence and key head is to be done again
  size_t bytes;
};

constexpr size_t kTileRecord = 52;
// Tiles of a head: a sequence ends at most one of them early.
__host__ inline size_t cache_max_tiles(const CacheGeom &g) { return (size_t)g.S + (size_t)g.T / (128 / g.G); }

__host__ inline CacheWorkspace carve_cache(const CacheGeom &g, void *base) {
  CacheWorkspace w;
  char *p = static_cast<char *>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char *at = p + off;
    off += align256(bytes);
    return at;
  };
  w.status = reinterpret_cast<int32_t *>(take(64 * sizeof(int32_t)));
  w.arrivals = reinterpret_cast<int32_t *>(take(2 * kCacheCtas * sizeof(int32_t)));
  w.found = reinterpret_cast<int *>(take(8 * kCacheCtas * sizeof(int)));
  w.parts = reinterpret_cast<float *>(take(sizeof(float) * 2 * kCacheCtas * 128 * kD));
  w.part_l = reinterpret_cast<float2 *>(take(sizeof(float2) * 2 * kCacheCtas * 128));
  w.tiles = take(kTileRecord * cache_max_tiles(g));
  w.tile_first = reinterpret_cast<long long *>(take(sizeof(long long) * (cache_max_tiles(g) + 1)));
  w.tile_head = reinterpret_cast<int *>(take(64 * sizeof(int)));
  w.cuts = reinterpret_cast<long long *>(take((kCacheCtas + 1) * sizeof(long long)));
  w.any_redo = reinterpret_cast<int *>(take(kCacheCtas * sizeof(int)));
  w.redo = reinterpret_cast<uint8_t *>(take((size_t)g.S * g.Hkv));
  w.bytes = off;
  return w;
}

int make_cache_geom(const heart_cache_config *c, CacheGeom *g);

cudaError_t launch_cache_write(const CacheGeom &g, const CacheIndex &ix, const void *K, const void *V, const heart_cache &c,
                               cudaStream_t s, int *launches);
cudaError_t launch_cache_read(const CacheGeom &g, const CacheIndex &ix, const heart_cache &c, void *K, void *V, cudaStream_t s,
                              int *launches);
// Attention by 8 or 16 query rows in registers, or by tiles of 128: the former where a sequence and key head has so few rows.  (20 sequences of 4000
// tokens, 32 heads on 8, bf16: four new tokens, 16 rows, 71 us; eight, 32 rows, 189 by rows and 75 by tiles.)
constexpr int kRowsOfRowsKernel = 16;
cudaError_t launch_cache_rows(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                              void *O, float *lse, cudaStream_t s, int *launches);
// Behind the tile kernel, for e4m3: by rows what `looked` CTAs have put down in w.redo (most often nothing).
cudaError_t launch_cache_redo(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                              void *O, float *lse, int looked, cudaStream_t s, int *launches);
cudaError_t launch_cache_tiles(const CacheGeom &g, const CacheIndex &ix, const CacheWorkspace &w, const void *Q, const heart_cache &c,
                               void *O, float *lse, cudaStream_t s, int *launches);

// A pool as a tensor map: boxes of `rows` slots of one head (of bf16, `halves` halves of their 128 dims).
bool make_pool_map(CUtensorMap *m, const void *base, const CacheGeom &g, int rows, int halves);

#ifdef __CUDACC__
// A scale byte as a number: 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float cache_scale(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// Two codes as f16, and two fp32 numbers.
__device__ __forceinline__ uint32_t codes_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t high_codes_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The scale of a row of codes whose largest bf16 magnitude has the bits `top`, as heart_cache_write has it (from 2^-100 on), NaN where
// that is not finite; inv: one over it.
__device__ __forceinline__ float code_scale(uint32_t top, float &inv) {
  const int e = min(max((int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u ? 1 : 0), -100), 120);
  inv = __uint_as_float((uint32_t)(127 - e) << 23);
  return __uint_as_float(top < 0x7f80u ? (uint32_t)(127 + e) << 23 : 0x7fc00000u);
}
// Two bf16 numbers times inv (a power of two that makes them 448 at most) as the sums of two e4m3 codes each: the codes nearest to them,
// and to what is left.  In f16, which holds the products but for bits below 2^-24, and the differences.
__device__ __forceinline__ void split_codes(uint32_t w, float inv, uint32_t &high, uint32_t &low) {
  const uint32_t x = pack_f16x2(__uint_as_float(w << 16) * inv, __uint_as_float(w & 0xffff0000u) * inv);
  uint16_t c;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
  high = c;
  uint32_t left;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(left) : "r"(x), "r"(codes_to_f16x2(high)));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(left));
  low = c;
}
// A sequence as its arrays describe it, brought into range (and reported) where they do not hold what they should.
struct Sequence {
  int row, n, len;  // first row, new tokens, tokens
};
__device__ __forceinline__ Sequence sequence(const CacheIndex &ix, int s) {
  int r0 = __ldcg(&ix.row_start[s]), r1 = __ldcg(&ix.row_start[s + 1]), len = __ldcg(&ix.kv_len[s]);
  const int most = ix.table_stride << ix.page_log2;
  if (r0 < 0 || r1 < r0 || r1 > ix.T || len < 0 || len > most) {
    atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
    r0 = min(max(r0, 0), ix.T);
    r1 = min(max(r1, r0), ix.T);
    len = min(max(len, 0), most);
  }
  return {r0, r1 - r0, len};
}
// The table's entry for token j < len of sequence s, and the page that it stands for: n_pages (reported) where it is none.  (Apart, so that
// an entry can be asked for ahead of its use.)
__device__ __forceinline__ int page_entry(const CacheIndex &ix, int s, int j) {
  return __ldcg(&ix.table[(size_t)s * ix.table_stride + (j >> ix.page_log2)]);
}
__device__ __forceinline__ int checked_page(const CacheIndex &ix, int page) {
  if ((unsigned)page < (unsigned)ix.n_pages) return page;
  atomicExch(ix.status, HEART_ERR_DEVICE_CHECK);
  return ix.n_pages;
}
__device__ __forceinline__ int page_of(const CacheIndex &ix, int s, int j) { return checked_page(ix, page_entry(ix, s, j)); }
// Visible keys of the query at position p of a sequence of `len` tokens: [low, end) and [0, sink).
struct Visible {
  int low, end;
};
__device__ __forceinline__ Visible visible(const CacheIndex &ix, int p, int len) {
  if (p < 0) return {0, 0};
  int end = len;
  if (ix.causal > 0) {
    const int group = p - p % ix.causal;
    end = ix.causal < len - group ? group + ix.causal : len;
  }
  return {ix.window > 0 && ix.window < end ? end - ix.window : 0, end};
}
// Key steps that the queries at positions p0 .. p1 see some key of: `sinks` steps from token 0 on, then those from step `first` on.
// (One step without any visible key where there is none, so that the rows are written.)
template <int Step = kKeyStep>
struct Span {
  int sinks, first, steps;
  __device__ __forceinline__ int step(int i) const { return i < sinks ? i : first + i - sinks; }
};
template <int Step = kKeyStep>
__device__ __forceinline__ Span<Step> span_of(const CacheIndex &ix, int p0, int p1, int len) {
  const Visible a = visible(ix, max(p0, 0), len), b = visible(ix, p1, len);
  if (p1 < 0 || b.end <= 0) return {0, 0, 1};
  Span<Step> r;
  r.first = a.low / Step;
  r.sinks = min((min(ix.sink, a.low) + Step - 1) / Step, r.first);
  r.steps = r.sinks + (b.end + Step - 1) / Step - r.first;
  return r;
}
#endif

}  // namespace heart
