// The 16 x 16 matrix product of rows as lanes load them, 16 bytes each, for products
// whose operands are not copied to LDS.
#pragma once
#include "vec_io.h"

namespace kkm {

typedef float floatx4 __attribute__((ext_vector_type(4)));

// The products of 16 bytes of each row: a lane's elements of row lane % 16 at
// k = kVec * (lane / 16) + e.  fp32: four instructions of 4 k each, one per e.
__device__ inline floatx4 mfma_few(raw_vec<float> a, raw_vec<float> b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ inline floatx4 mfma_few(raw_vec<half_t> a, raw_vec<half_t> b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline floatx4 mfma_few(raw_vec<bf16_t> a, raw_vec<bf16_t> b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

}  // namespace kkm
