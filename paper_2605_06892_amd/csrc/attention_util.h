// Device helpers shared by the attention kernels.
#pragma once

#include "common.h"

namespace hsa {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
// fp32 rows are only 4-byte aligned
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// The W x W fp32 matrix instruction: 64/W contraction slots (lane / W), the
// result's column lane % W, its rows row(e, lane / W) for e < W*W/64.
template <int W>
struct Mfma;
template <>
struct Mfma<32> {
  typedef f32x16 acc;
  static __device__ __forceinline__ acc mul(float a, float b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ int row(int e, int slot) { return (e >> 2) * 8 + slot * 4 + (e & 3); }
};
template <>
struct Mfma<16> {
  typedef f32x4 acc;
  static __device__ __forceinline__ acc mul(float a, float b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ int row(int e, int slot) { return slot * 4 + e; }
};

// exp(x) for x <= 0 (NaN stays NaN): 2^t with t = fl(x log2 e), corrected by
// the remainder x - t ln 2, which is exact to below an ulp. Results under 2^-126,
// which v_exp_f32 flushes (expf does not), are 0: a key's weight of 1e-38 of the greatest.
__device__ __forceinline__ float exp_neg(float x) {
  const float c = x < -104.f ? -104.f : x;
  const float t = c * 1.44269504088896341f;
  const float e = __builtin_amdgcn_exp2f(t);
  const float u = fmaf(-t, -1.90465429995776804525e-09f, fmaf(-t, 0.693147182464599609375f, c));
  return fmaf(e, u, e);
}

}  // namespace hsa
