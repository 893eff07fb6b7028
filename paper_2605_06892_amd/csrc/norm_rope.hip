// RMS norms of the heads of queries and keys, and their rotation by position, in one pass:
//   y = x / sqrt(mean x^2 + eps) * weight,   (a, b) -> (a cos - b sin, a sin + b cos)
// for the pairs of the first rope_dim channels, rounded once. A stream: every value is
// read and written once, 8 per thread; head_dim / 8 neighbouring lanes share a head and its sum.
// Pairs of neighbouring channels lie in one lane. For pairs (c, c + rope_dim / 2) a lane takes
// 4 channels of either half, so that they do too.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;

template <bool BF16>
struct Four;  // 4 neighbouring values
template <>
struct Four<true> {
  typedef bf16x4 T;
  static __device__ __forceinline__ f32x4 load(const void* p, long i) {
    return __builtin_convertvector(*reinterpret_cast<const bf16x4*>(static_cast<const bf16*>(p) + i), f32x4);
  }
  static __device__ __forceinline__ void store(void* p, long i, f32x4 x) {
    *reinterpret_cast<bf16x4*>(static_cast<bf16*>(p) + i) = to_bf16x4(x);
  }
};
template <>
struct Four<false> {
  static __device__ __forceinline__ f32x4 load(const void* p, long i) {
    return *reinterpret_cast<const f32x4u*>(static_cast<const float*>(p) + i);
  }
  static __device__ __forceinline__ void store(void* p, long i, f32x4 x) {
    *reinterpret_cast<f32x4u*>(static_cast<float*>(p) + i) = x;
  }
};

// sum over the L lanes (8 or 16, aligned) of a head, the same in all of them
template <int L>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) x += __shfl_xor(x, o);
  return x;
}
template <int L>
__device__ __forceinline__ double head_sum(double x) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

template <bool BF16, int DH>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRope a, FastDiv all_heads) {
  constexpr int L = DH / 8;
  const int lane = threadIdx.x % L;
  const long unit = (long)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const long row = unit / all_heads.d;
  if (row >= a.n) return;
  int h = (int)(unit - row * all_heads.d);
  const bool is_q = h < a.heads;
  if (!is_q) h -= a.heads;
  const void* src = is_q ? a.q : a.k;
  void* dst = is_q ? a.q_out : a.k_out;
  const void* weight = is_q ? a.q_weight : a.k_weight;
  const long from = row * (is_q ? a.q_stride : a.k_stride) + h * DH, to = row * (is_q ? a.qo_stride : a.ko_stride) + h * DH;

  // this lane's channels c0 .. c0+3 and c1 .. c1+3, and its first pair
  int c0 = lane * 8, c1 = c0 + 4, pair = lane * 4;
  if (!a.interleaved) {
    const int half = a.rope_dim / 2;
    c0 = pair < half ? pair : pair + half;
    c1 = c0 + (pair < half ? half : (DH - a.rope_dim) / 2);
  }
  f32x4 x = Four<BF16>::load(src, from + c0), y = Four<BF16>::load(src, from + c1);
  f32x4 wx = {1.f, 1.f, 1.f, 1.f}, wy = wx;
  if (weight) {
    wx = Four<BF16>::load(weight, c0);
    wy = Four<BF16>::load(weight, c1);
  }
  f32x4 cs[2] = {{1.f, 0.f, 1.f, 0.f}, {1.f, 0.f, 1.f, 0.f}};
  if (pair < a.rope_dim / 2) {
    const long p = a.pos ? a.pos[row] : row;
    if (p >= 0 && p < a.n_pos) {
      const f32x4* t = reinterpret_cast<const f32x4*>(a.rope + p * a.rope_dim + pair * 2);
      cs[0] = t[0];
      cs[1] = t[1];
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum = fmaf(x[j], x[j], fmaf(y[j], y[j], sum));
  sum = head_sum<L>(sum);
  float f = 1.f / sqrtf(sum * (1.f / DH) + a.eps);
  // squares past fp32, or all of them so small that bits are lost beside a smaller eps: in 64 bits
  const bool far = sum > 0x1p125f || (sum < 0x1p-90f && a.eps < 0x1p-80f);
  if (__any(far)) {
    double s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) s += (double)x[j] * x[j] + (double)y[j] * y[j];
    s = 1.0 / sqrt(head_sum<L>(s) / DH + a.eps);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (far) x[j] = (float)(x[j] * s), y[j] = (float)(y[j] * s);
    }
    if (far) f = 1.f;
  }
  x = x * f * wx;
  y = y * f * wy;
  f32x4 u, v;
  if (a.interleaved) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x2 p = rope_rotate((f32x2){cs[0][2 * j], cs[0][2 * j + 1]}, x[2 * j], x[2 * j + 1]);
      const f32x2 q = rope_rotate((f32x2){cs[1][2 * j], cs[1][2 * j + 1]}, y[2 * j], y[2 * j + 1]);
      u[2 * j] = p[0], u[2 * j + 1] = p[1], v[2 * j] = q[0], v[2 * j + 1] = q[1];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 p = rope_rotate((f32x2){cs[j >> 1][2 * (j & 1)], cs[j >> 1][2 * (j & 1) + 1]}, x[j], y[j]);
      u[j] = p[0], v[j] = p[1];
    }
  }
  Four<BF16>::store(dst, to + c0, u);
  Four<BF16>::store(dst, to + c1, v);
}

template <bool BF16, int DH>
hipError_t launch(const NormRope& a, hipStream_t s) {
  constexpr int per = kThreads / (DH / 8);
  const uint32_t heads = (uint32_t)(a.heads + a.kv_heads);
  const long groups = ((long)a.n * heads + per - 1) / per;
  hipLaunchKernelGGL((norm_rope_kernel<BF16, DH>), dim3((unsigned)groups), dim3(kThreads), 0, s, a, FastDiv(heads));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope(const NormRope& a, bool bf16, int head_dim, hipStream_t s) {
  if (a.n <= 0 || a.heads + a.kv_heads <= 0) return hipSuccess;
  if (bf16) return head_dim == 64 ? launch<true, 64>(a, s) : launch<true, 128>(a, s);
  return head_dim == 64 ? launch<false, 64>(a, s) : launch<false, 128>(a, s);
}

}  // namespace hsa
