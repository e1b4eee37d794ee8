// What the kernels that work on tiles of 128 packed query rows share.
#pragma once
#include "cache.cuh"
#include "tc_ptx.cuh"

namespace heart {
namespace tc {

__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// Weights 2^(s*c - m) of 32 scores of a row, packed to bf16 or f16, and their sums (of the weights before they are rounded: the log-sum-exp
// is then good to 32 bits).
template <bool F16>
__device__ __forceinline__ void exp32(const uint32_t *s, uint64_t c2, uint64_t neg_m2, uint32_t *pk, uint64_t (&sums)[2]) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    float x0, x1, x2, x3;
    unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2, neg_m2), x0, x1);
    unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), c2, neg_m2), x2, x3);
    x0 = ex2(x0), x1 = ex2(x1), x2 = ex2(x2), x3 = ex2(x3);
    sums[0] = add_f32x2(sums[0], pack_f32x2(x0, x1));
    sums[1] = add_f32x2(sums[1], pack_f32x2(x2, x3));
    pk[i >> 1] = F16 ? pack_f16x2(x0, x1) : pack_bf16x2(x0, x1);
    pk[(i >> 1) + 1] = F16 ? pack_f16x2(x2, x3) : pack_bf16x2(x2, x3);
  }
}
__device__ __forceinline__ void sts_u4(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Q as (64 dims, query head of its key head, token, dim half, key head): a box is the tokens of a tile with their G heads.
template <typename G>
bool make_query_map(CUtensorMap *m, const void *Q, const G &g) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[5] = {64, (cuuint64_t)g.G, (cuuint64_t)g.T, 2, (cuuint64_t)g.Hkv};
  cuuint64_t strides[4] = {(cuuint64_t)g.qh * 2, (cuuint64_t)g.qt * 2, 128, (cuuint64_t)g.qh * g.G * 2};
  cuuint32_t box[5] = {64, (cuuint32_t)g.G, (cuuint32_t)(128 / g.G), 1, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(Q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace heart
