// Rows times weights in e2m1 groups: y = act(s (x W^T)) + r for a few rows, bound by reading W.
//
// A wave takes 16 outputs (the rows of the matrix instructions' tile) and 128 inputs of W at a
// time: each lane loads 16 bytes, the 32 codes of one group, and that group's exponent, which
// the conversion to bf16 takes as its operand: exact, one instruction for two weights, and no
// scaling of sums. Slot lane / 16 of the contraction holds that group, 8 values to an instruction, so
// x is read in the same order. The rows of x are the tile's columns, 16 to a tile.
// The waves of a workgroup take 128 inputs each in turn and are joined in LDS.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kOuts = 16;   // outputs of a tile, and rows of x of one
constexpr int kStep = 128;  // inputs of a wave's load
constexpr int kWaves = 8;

__device__ __forceinline__ float gelu_exact(float x) {
  const float y = 0.7978845608028654f * fmaf(0.044715f * x, x * x, x);
  return x / (1.f + expf(-2.f * y));
}

// 8 codes of a word as bf16, times 2^e in `scale`
__device__ __forceinline__ bf16x8 widen8(unsigned c, float scale) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
  return (bf16x8){p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
}

template <bool BF16, int NT>
__global__ __launch_bounds__(kWaves * kWave) void linear_w4_kernel(LinearW4 a) {
  __shared__ __attribute__((aligned(16))) f32x4 parts[kWaves][NT][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int l16 = lane & 15, grp = lane >> 4;
  const int o0 = blockIdx.x * kOuts, m0 = blockIdx.y * (kOuts * NT);
  const long w_row = min(o0 + l16, a.d_out - 1);
  const uint8_t* w = a.w + w_row * (a.d_in / 2);
  const int8_t* e = a.exps + w_row * (a.d_in / kGroup);
  long x_row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x_row[t] = (long)min(m0 + t * kOuts + l16, a.rows - 1) * a.d_in;

  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = (f32x4){};
  for (int k0 = wave * kStep; k0 < a.d_in; k0 += kWaves * kStep) {
    const int k = k0 + grp * kGroup;
    const bool in = k < a.d_in;  // the last step may have fewer groups: 0 times 0
    u32x4 c = {};
    float s = 1.f;
    if (in) {
      c = *reinterpret_cast<const u32x4*>(w + k / 2);
      s = pow2(e[k / kGroup]);
    }
    if constexpr (BF16) {
      bf16x8 x[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[t][i] = (bf16x8){};
          if (in) x[t][i] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.x) + x_row[t] + k + i * 8);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 y = widen8(c[i], s);
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x[t][i], acc[t], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 x[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            x[t][j] = (f32x4){};
            if (in) x[t][j] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.x) + x_row[t] + k + i * 8 + j * 4);
          }
        const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 0), q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 1);
        const f32x2 r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 2), u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 3);
        const float y[8] = {p[0], p[1], q[0], q[1], r[0], r[1], u[0], u[1]};
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t] = Mfma<16>::mul(y[j], x[t][j >> 2][j & 3], acc[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) parts[wave][t][lane] = acc[t];
  __syncthreads();
  // acc[e] of a lane: output o0 + grp * 4 + e of row l16 of the tile
  for (int f = threadIdx.x; f < NT * kWave; f += kWaves * kWave) {
    const int t = f / kWave, l = f % kWave;
    const int m = m0 + t * kOuts + (l & 15), o = o0 + (l >> 4) * 4;
    if (m >= a.rows) continue;
    f32x4 sum = parts[0][t][l];
#pragma unroll
    for (int x = 1; x < kWaves; ++x) sum += parts[x][t][l];
    if (a.row_scale) sum *= a.row_scale[m];
    const long at = (long)m * a.d_out + o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.d_out) break;
      float z = sum[j];
      if constexpr (BF16) {
        if (a.gelu) z = gelu_tanh(z);
        if (a.residual) z += (float)static_cast<const bf16*>(a.residual)[at + j];
        if (a.out_f32) static_cast<float*>(a.y)[at + j] = z;
        else static_cast<bf16*>(a.y)[at + j] = (bf16)z;
      } else {
        if (a.gelu) z = gelu_exact(z);
        if (a.residual) z += static_cast<const float*>(a.residual)[at + j];
        static_cast<float*>(a.y)[at + j] = z;
      }
    }
  }
}

template <bool BF16, int NT>
hipError_t launch(const LinearW4& a, hipStream_t s) {
  const unsigned outs = (unsigned)((a.d_out + kOuts - 1) / kOuts), rows = (unsigned)((a.rows + NT * kOuts - 1) / (NT * kOuts));
  hipLaunchKernelGGL((linear_w4_kernel<BF16, NT>), dim3(outs, rows), dim3(kWaves * kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_w4(const LinearW4& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0 || a.d_out <= 0) return hipSuccess;
  if (bf16) return a.rows <= 16 ? launch<true, 1>(a, s) : a.rows <= 32 ? launch<true, 2>(a, s) : launch<true, 4>(a, s);
  return a.rows <= 16 ? launch<false, 1>(a, s) : launch<false, 2>(a, s);
}

}  // namespace hsa
