// Storing new tokens' keys and values in their pages, as they are or quantised, and reading tokens back.
//
// Both move rows of 128 elements, one token of one key head, and nothing is used twice: HBM bounds them.  A warp takes one
// token and kHeads heads: lanes 0-15 its keys, lanes 16-31 its values, 16 bytes of bf16 a lane.  The way to the token's slot is a chain of
// three loads (sequence, length, page).  A write asks for its rows before it goes that way; a read needs the way first, so it relies on
// many warps an SM.
//
// e4m3: the scale is a power of two, so that x * 2^-e and code * 2^e are exact and the code's rounding (to nearest even, by
// the conversion instruction) is the only one: half a step, 2^-4 of a value from 2^(e-6) on, 2^(e-10) below.
#include "cache.cuh"

namespace heart {
namespace {

constexpr int kHeads = 4;    // heads a warp takes
constexpr int kWarps = 8;    // a CTA
constexpr int kMaxExponent = 120;   // of a scale: the largest bf16 number is below 448 * 2^120
constexpr int kMinExponent = -110;  // keeps every code times its scale a normal fp32 number

struct CopyParams {
  CacheIndex ix;
  const uint16_t *K, *V;     // packed rows (write)
  uint16_t *K_out, *V_out;   // packed rows (read)
  unsigned char *k, *v;      // pools
  uint8_t *k_scale, *v_scale;
  long long kvt, kvh, pp, ph, pt;
  int Hkv, groups;           // groups of kHeads heads
};

// The sequence of row `row`, or -1: rows of no sequence.  32 places of row_start at a time, the whole warp.
__device__ __forceinline__ int sequence_of(const CacheIndex &ix, int row, int lane) {
  int lo = 0, hi = ix.S;  // row_start[lo] <= row < row_start[hi], if row belongs to a sequence
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + lane * step;
    const bool below = at < hi && (lane == 0 || __ldcg(&ix.row_start[at]) <= row);
    const int n = __popc(__ballot_sync(0xffffffffu, below));  // (ascending: a run of lanes from 0 on)
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// The token's slot as an offset in elements (heads apart) and its number among the scales; false: there is none.
__device__ __forceinline__ bool slot_of(const CopyParams &p, int row, int lane, bool &belongs, long long &at, long long &scale_at) {
  const int s = sequence_of(p.ix, row, lane);
  const Sequence q = sequence(p.ix, s);
  belongs = row >= q.row && row < q.row + q.n;
  const int pos = q.len - q.n + (row - q.row);
  if (!belongs || pos < 0) return false;
  const int page = page_of(p.ix, s, pos), slot = pos & ((1 << p.ix.page_log2) - 1);
  if (page == p.ix.n_pages) return false;
  at = (long long)page * p.pp + (long long)slot * p.pt;
  scale_at = ((long long)page * p.Hkv << p.ix.page_log2) + slot;
  return true;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

__device__ __forceinline__ float bf16_low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

__device__ __forceinline__ uint32_t to_e4m3x2(uint32_t x, float inv, float most) {
  const float lo = fminf(fmaxf(bf16_low(x) * inv, -most), most), hi = fminf(fmaxf(bf16_high(x) * inv, -most), most);
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool E4m3>
__global__ void __launch_bounds__(32 * kWarps) cache_write_kernel(const CopyParams p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int row = (int)(warp / p.groups), h0 = (int)(warp % p.groups) * kHeads;
  pdl_wait();
  pdl_launch_dependents();
  if (row >= p.ix.T) return;
  const bool values = lane >= 16;
  const int i = lane & 15;
  const uint16_t *src = (values ? p.V : p.K) + row * p.kvt + i * 8;
  uint4 x[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u)
    x[u] = h0 + u < p.Hkv ? __ldcs(reinterpret_cast<const uint4 *>(src + (h0 + u) * p.kvh)) : make_uint4(0u, 0u, 0u, 0u);
  bool belongs;
  long long at, scale_at;
  if (!slot_of(p, row, lane, belongs, at, scale_at)) return;
  unsigned char *pool = values ? p.v : p.k;
  uint8_t *scales = values ? p.v_scale : p.k_scale;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (h0 + u >= p.Hkv) break;
    const long long to = at + (h0 + u) * p.ph + i * 8;
    if (!E4m3) {
      *reinterpret_cast<uint4 *>(pool + 2 * to) = x[u];
      continue;
    }
    // the largest magnitude of the row: bf16 magnitudes compare as whole numbers
    uint32_t top = max_u16x2(max_u16x2(x[u].x & 0x7fff7fffu, x[u].y & 0x7fff7fffu), max_u16x2(x[u].z & 0x7fff7fffu, x[u].w & 0x7fff7fffu));
    top = max(top & 0xffffu, top >> 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // top = 1.m * 2^(field - 127); 448 = 1.75 * 2^8
    const int e = max((int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u ? 1 : 0), kMinExponent);
    const bool finite = top < 0x7f80u;
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint2 code = make_uint2(0u, 0u);
    const float most = e < kMaxExponent ? 448.f : 240.f;  // (256 * 2^120 is no bf16 number)
    if (finite) {
      code.x = to_e4m3x2(x[u].x, inv, most) | to_e4m3x2(x[u].y, inv, most) << 16;
      code.y = to_e4m3x2(x[u].z, inv, most) | to_e4m3x2(x[u].w, inv, most) << 16;
    }
    *reinterpret_cast<uint2 *>(pool + to) = code;
    if (i == 0) scales[scale_at + ((long long)(h0 + u) << p.ix.page_log2)] = (uint8_t)(finite ? e + 127 : 255);
  }
}

// Two codes times 2^(scale byte - 127), as bf16: exact (see heart_cache_write).
__device__ __forceinline__ uint32_t from_e4m3x2(uint32_t codes, float scale) {
  // sign, exponent and mantissa at their places in bf16, with the exponent field 120 too small
  const uint32_t x = __byte_perm(codes, 0, 0x1404);
  const uint32_t t = ((x >> 4) & 0x07f007f0u) | (x & 0x80008000u);
  const float lo = bf16_low(t) * 0x1p120f * scale, hi = bf16_high(t) * 0x1p120f * scale;
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}

template <bool E4m3>
__global__ void __launch_bounds__(32 * kWarps) cache_read_kernel(const CopyParams p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int row = (int)(warp / p.groups), h0 = (int)(warp % p.groups) * kHeads;
  pdl_wait();
  pdl_launch_dependents();
  if (row >= p.ix.T) return;
  const bool values = lane >= 16;
  const int i = lane & 15;
  bool belongs;
  long long at = 0, scale_at = 0;
  const bool there = slot_of(p, row, lane, belongs, at, scale_at);
  if (!belongs) return;
  const unsigned char *pool = values ? p.v : p.k;
  const uint8_t *scales = values ? p.v_scale : p.k_scale;
  uint16_t *out = (values ? p.V_out : p.K_out) + row * p.kvt + i * 8;
  uint4 x[kHeads];
  uint32_t b[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    x[u] = make_uint4(0u, 0u, 0u, 0u);
    b[u] = 127u;
    if (there && h0 + u < p.Hkv) {
      const long long from = at + (h0 + u) * p.ph + i * 8;
      if (E4m3) {
        const uint2 c = __ldcs(reinterpret_cast<const uint2 *>(pool + from));
        x[u].x = c.x;
        x[u].y = c.y;
        b[u] = scales[scale_at + ((long long)(h0 + u) << p.ix.page_log2)];
      } else {
        x[u] = __ldcs(reinterpret_cast<const uint4 *>(pool + 2 * from));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (h0 + u >= p.Hkv) break;
    if (E4m3) {
      const float scale = cache_scale(b[u]);
      const uint2 c = make_uint2(x[u].x, x[u].y);
      x[u] = make_uint4(from_e4m3x2(c.x & 0xffffu, scale), from_e4m3x2(c.x >> 16, scale), from_e4m3x2(c.y & 0xffffu, scale),
                        from_e4m3x2(c.y >> 16, scale));
    }
    __stcs(reinterpret_cast<uint4 *>(out + (h0 + u) * p.kvh), x[u]);
  }
}

CopyParams copy_params(const CacheGeom &g, const CacheIndex &ix, const heart_cache &c) {
  CopyParams p = {};
  p.ix = ix;
  p.k = static_cast<unsigned char *>(c.k);
  p.v = static_cast<unsigned char *>(c.v);
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.kvt = g.kvt;
  p.kvh = g.kvh;
  p.pp = g.pp;
  p.ph = g.ph;
  p.pt = g.pt;
  p.Hkv = g.Hkv;
  p.groups = (g.Hkv + kHeads - 1) / kHeads;
  return p;
}

template <typename K>
cudaError_t launch_copy(K *kernel, const CopyParams &p, cudaStream_t s, int *launches) {
  const long long warps = (long long)p.ix.T * p.groups;
  ++*launches;
  return launch_pdl(kernel, dim3((unsigned)((warps + kWarps - 1) / kWarps)), dim3(32 * kWarps), 0, s, p);
}

}  // namespace

cudaError_t launch_cache_write(const CacheGeom &g, const CacheIndex &ix, const void *K, const void *V, const heart_cache &c,
                               cudaStream_t s, int *launches) {
  CopyParams p = copy_params(g, ix, c);
  p.K = static_cast<const uint16_t *>(K);
  p.V = static_cast<const uint16_t *>(V);
  return launch_copy(g.e4m3 ? cache_write_kernel<true> : cache_write_kernel<false>, p, s, launches);
}

cudaError_t launch_cache_read(const CacheGeom &g, const CacheIndex &ix, const heart_cache &c, void *K, void *V, cudaStream_t s,
                              int *launches) {
  CopyParams p = copy_params(g, ix, c);
  p.K_out = static_cast<uint16_t *>(K);
  p.V_out = static_cast<uint16_t *>(V);
  return launch_copy(g.e4m3 ? cache_read_kernel<true> : cache_read_kernel<false>, p, s, launches);
}

}  // namespace heart
