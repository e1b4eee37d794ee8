// Storing new tokens' keys and values in their pages, as they are or quantised, and reading tokens back.
//
// Both move rows of 128 elements, one token of one key head, and nothing is used twice: HBM bounds them, and next to it the
// instructions of the conversion.  A warp takes one token and a range of heads: lanes 0-15 its keys, lanes 16-31 its values, eight lanes a row, two
// pieces of 16 bytes (of bf16) a lane, so that what is done once a row (the largest magnitude over its lanes, the scale) is done for two
// heads at once.  The way to the token's slot is a chain of three loads (sequence, length, page); a write asks for its first rows before it
// goes that way.  Heads are shared among as many warps as make some waves of all SMs.
//
// e4m3: the scale is a power of two, so that x * 2^-e and code * 2^e are exact and the code's rounding (to nearest even, by
// the conversion instruction) is the only one: half a step, 2^-4 of a value from 2^(e-6) on, 2^(e-10) below.
#include "cache.cuh"

namespace heart {
namespace {

constexpr int kUnroll = 2;   // pairs of heads a warp has in flight
constexpr int kWarps = 8;    // a CTA
constexpr int kWantedWarps = 148 * 48 * 4;
constexpr int kMaxExponent = 120;   // of a scale: the largest bf16 number is below 448 * 2^120
constexpr int kMinExponent = -110;  // keeps every code times its scale a normal fp32 number

struct CopyParams {
  CacheIndex ix;
  const uint16_t *K, *V;     // packed rows (write)
  uint16_t *K_out, *V_out;   // packed rows (read)
  unsigned char *k, *v;      // pools
  uint8_t *k_scale, *v_scale;
  long long kvt, kvh, pp, ph, pt;
  int Hkv, heads;            // of a warp
};

// The sequence of row `row` if it belongs to one.  32 places of row_start at a time, the whole warp; up to 32 sequences are asked for as they are,
// which saves a trip.
__device__ __forceinline__ Sequence sequence_of(const CacheIndex &ix, int row, int lane, int &s) {
  if (ix.S <= 32) {
    const Sequence q = sequence(ix, min(lane, ix.S - 1));
    s = __popc(__ballot_sync(0xffffffffu, lane < ix.S && q.row <= row)) - 1;  // (ascending: a run of lanes from 0 on)
    s = max(s, 0);
    return {__shfl_sync(0xffffffffu, q.row, s), __shfl_sync(0xffffffffu, q.n, s), __shfl_sync(0xffffffffu, q.len, s)};
  }
  int lo = 0, hi = ix.S;  // row_start[lo] <= row < row_start[hi], if row belongs to a sequence
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + lane * step;
    const bool below = at < hi && (lane == 0 || __ldcg(&ix.row_start[at]) <= row);
    const int n = __popc(__ballot_sync(0xffffffffu, below));
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  s = lo;
  return sequence(ix, s);
}

// More than 32 sequences: all of them looked at, each by one thread of the launch (a row's way to its slot passes a few).
__device__ __forceinline__ void check_sequences(const CacheIndex &ix) {
  if (ix.S <= 32) return;
  const long long threads = (long long)gridDim.x * gridDim.y * blockDim.x;
  for (long long s = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x; s < ix.S; s += threads) sequence(ix, (int)s);
}

// The token's slot as an offset in elements (heads apart) and its number among the scales; false: there is none.
__device__ __forceinline__ bool slot_of(const CopyParams &p, int row, int lane, bool &belongs, long long &at, long long &scale_at) {
  int s;
  const Sequence q = sequence_of(p.ix, row, lane, s);
  belongs = row >= q.row && row < q.row + q.n;
  const int pos = q.len - q.n + (row - q.row);
  if (!belongs || pos < 0) return false;
  const int page = page_of(p.ix, s, pos), slot = pos & ((1 << p.ix.page_log2) - 1);
  if (page == p.ix.n_pages) return false;
  at = (long long)page * p.pp + (long long)slot * p.pt;
  scale_at = ((long long)page * p.Hkv << p.ix.page_log2) + slot;
  return true;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// 2^e as bf16, twice
__device__ __forceinline__ uint32_t power_bf16x2(int e) { return (uint32_t)(e + 127) * 0x00800080u; }

__device__ __forceinline__ uint32_t to_e4m3x2(uint32_t x) {  // two bf16 numbers
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__uint_as_float(x & 0xffff0000u)), "f"(__uint_as_float(x << 16)));
  return r;
}
__device__ __forceinline__ uint2 to_codes(const uint4 &x, uint32_t inv) {  // eight elements times inv
  return make_uint2(to_e4m3x2(mul_bf16x2(x.x, inv)) | to_e4m3x2(mul_bf16x2(x.y, inv)) << 16,
                    to_e4m3x2(mul_bf16x2(x.z, inv)) | to_e4m3x2(mul_bf16x2(x.w, inv)) << 16);
}
__device__ __forceinline__ uint32_t largest(const uint4 &x) {  // of both halves: bf16 magnitudes compare as whole numbers
  return __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}
// Magnitudes above 240 * 2^120 as that: 256 * 2^120 is no bf16 number.
__device__ __forceinline__ uint32_t below_256(uint32_t x) { return (x & 0x80008000u) | __vminu2(x & 0x7fff7fffu, 0x7f707f70u); }

template <bool E4m3>
__global__ void __launch_bounds__(32 * kWarps) cache_write_kernel(const CopyParams p) {
  const int lane = threadIdx.x & 31, row = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int values = lane >> 4, i = lane & 7;
  int h = blockIdx.y * p.heads + ((lane >> 3) & 1);
  const int h1 = min(p.Hkv, (int)(blockIdx.y + 1) * p.heads), count = h1 - (int)blockIdx.y * p.heads;
  pdl_wait();
  pdl_launch_dependents();
  check_sequences(p.ix);
  if (row >= p.ix.T) return;
  const uint16_t *src = (values ? p.V : p.K) + row * p.kvt + h * p.kvh + i * 8;
  uint4 x[kUnroll][2];
  auto load = [&]() {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        x[u][k] = h + 2 * u < h1 ? __ldcs(reinterpret_cast<const uint4 *>(src + 2 * u * p.kvh + k * 64)) : make_uint4(0u, 0u, 0u, 0u);
    src += 2 * kUnroll * p.kvh;
  };
  load();
  bool belongs;
  long long at, scale_at;
  if (!slot_of(p, row, lane, belongs, at, scale_at)) return;
  unsigned char *to = (values ? p.v : p.k) + (at + h * p.ph + i * 8) * (E4m3 ? 1 : 2);
  uint8_t *scale = E4m3 ? (values ? p.v_scale : p.k_scale) + scale_at + ((long long)h << p.ix.page_log2) : nullptr;
#pragma unroll 1
  for (int done = 0; done < count; done += 2 * kUnroll) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool there = h + 2 * u < h1;
      if (!E4m3) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (there) *reinterpret_cast<uint4 *>(to + 2 * (2 * u * p.ph + k * 64)) = x[u][k];
        continue;
      }
      uint32_t top = __vmaxu2(largest(x[u][0]), largest(x[u][1]));
      top = max(top & 0xffffu, top >> 16);
#pragma unroll
      for (int o = 4; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      // top = 1.m * 2^(field - 127); 448 = 1.75 * 2^8
      const int e = max((int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u ? 1 : 0), kMinExponent);
      if (e == kMaxExponent) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          x[u][k] = make_uint4(below_256(x[u][k].x), below_256(x[u][k].y), below_256(x[u][k].z), below_256(x[u][k].w));
      }
      const bool finite = top < 0x7f80u;
      const uint32_t inv = finite ? power_bf16x2(-e) : 0u;
      if (there) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint2 code = to_codes(x[u][k], inv);
          *reinterpret_cast<uint2 *>(to + 2 * u * p.ph + k * 64) = finite ? code : make_uint2(0u, 0u);
        }
        if (i == 0) scale[2 * u << p.ix.page_log2] = (uint8_t)(finite ? e + 127 : 255);
      }
    }
    h += 2 * kUnroll;
    to += 2 * kUnroll * p.ph * (E4m3 ? 1 : 2);
    if (E4m3) scale += 2 * kUnroll << p.ix.page_log2;
    if (done + 2 * kUnroll < count) load();
  }
}

// Four codes times 2^e as bf16, exact (see heart_cache_write): sign, exponent and mantissa are put at their places, with the exponent field
// 120 too small; f times rest, 2^(120 + e), sets that right.
__device__ __forceinline__ uint2 from_codes(uint32_t w, uint32_t f, uint32_t rest) {
  const uint32_t lo = __byte_perm(w, 0, 0x1404), hi = __byte_perm(w, 0, 0x3424);
  return make_uint2(mul_bf16x2(mul_bf16x2(((lo >> 4) & 0x07f007f0u) | (lo & 0x80008000u), f), rest),
                    mul_bf16x2(mul_bf16x2(((hi >> 4) & 0x07f007f0u) | (hi & 0x80008000u), f), rest));
}

template <bool E4m3>
__global__ void __launch_bounds__(32 * kWarps) cache_read_kernel(const CopyParams p) {
  const int lane = threadIdx.x & 31, row = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int values = lane >> 4, i = lane & 7;
  int h = blockIdx.y * p.heads + ((lane >> 3) & 1);
  const int h1 = min(p.Hkv, (int)(blockIdx.y + 1) * p.heads), count = h1 - (int)blockIdx.y * p.heads;
  pdl_wait();
  pdl_launch_dependents();
  check_sequences(p.ix);
  if (row >= p.ix.T) return;
  bool belongs;
  long long at = 0, scale_at = 0;
  const bool there = slot_of(p, row, lane, belongs, at, scale_at);
  if (!belongs) return;
  const unsigned char *from = (values ? p.v : p.k) + (at + h * p.ph + i * 8) * (E4m3 ? 1 : 2);
  const uint8_t *scale = E4m3 ? (values ? p.v_scale : p.k_scale) + scale_at + ((long long)h << p.ix.page_log2) : nullptr;
  uint16_t *out = (values ? p.V_out : p.K_out) + row * p.kvt + h * p.kvh + i * 8;
#pragma unroll 1
  for (int done = 0; done < count; done += 2 * kUnroll) {
    uint4 x[kUnroll][2];
    uint32_t b[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool some = there && h + 2 * u < h1;
      b[u] = 127u;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        x[u][k] = make_uint4(0u, 0u, 0u, 0u);
        if (E4m3) {
          if (some) {
            const uint2 c = __ldcs(reinterpret_cast<const uint2 *>(from + 2 * u * p.ph + k * 64));
            x[u][k].x = c.x;
            x[u][k].y = c.y;
          }
        } else {
          if (some) x[u][k] = __ldcs(reinterpret_cast<const uint4 *>(from + 2 * (2 * u * p.ph + k * 64)));
        }
      }
      if (E4m3 && some) b[u] = scale[2 * u << p.ix.page_log2];
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (h + 2 * u >= h1) break;
      if (E4m3) {
        const int e = (int)b[u] - 127;
        const uint32_t f = b[u] == 255u ? 0x7fc07fc0u : power_bf16x2(120 + min(e, 0)), rest = power_bf16x2(min(max(e, 0), 127));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint2 lo = from_codes(x[u][k].x, f, rest), hi = from_codes(x[u][k].y, f, rest);
          x[u][k] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) __stcs(reinterpret_cast<uint4 *>(out + 2 * u * p.kvh + k * 64), x[u][k]);
    }
    h += 2 * kUnroll;
    from += 2 * kUnroll * p.ph * (E4m3 ? 1 : 2);
    if (E4m3) scale += 2 * kUnroll << p.ix.page_log2;
    out += 2 * kUnroll * p.kvh;
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
  const long long shares = (kWantedWarps + (long long)g.T - 1) / g.T;
  p.heads = (int)max(4LL, (g.Hkv + shares - 1) / shares + 1 & ~1LL);  // (a warp goes by pairs, and the way to its slot is worth two of them)
  return p;
}

template <typename K>
cudaError_t launch_copy(K *kernel, const CopyParams &p, cudaStream_t s, int *launches) {
  ++*launches;
  return launch_pdl(kernel, dim3((p.ix.T + kWarps - 1) / kWarps, (p.Hkv + p.heads - 1) / p.heads), dim3(32 * kWarps), 0, s, p);
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
