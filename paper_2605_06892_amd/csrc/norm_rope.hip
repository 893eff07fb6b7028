// RMS norms of the heads of queries and keys, and their rotation by position, in one pass:
//   y = x / sqrt(mean x^2 + eps) * weight,   (a, b) -> (a cos - b sin, a sin + b cos)
// for the pairs of the first rope_dim channels, rounded once. A stream: every value is
// read and written once, 8 per thread and head; head_dim / 8 neighbouring lanes share a head and its sum.
// Pairs of neighbouring channels lie in one lane. For pairs (c, c + rope_dim / 2) a lane takes
// 4 channels of either half, so that they do too.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;

// A lane's 8 values: two runs of 4, at c0 and c1 = c0 + 4 (NEAR: one load) or c1 anywhere. Stores of a large launch
// (PAST) pass the caches by.
template <bool PAST, class T>
__device__ __forceinline__ void put(T x, void* p) {
  if constexpr (PAST) __builtin_nontemporal_store(x, static_cast<T*>(p));
  else *static_cast<T*>(p) = x;
}
template <bool BF16, bool NEAR, bool PAST>
struct Eight {
  static __device__ __forceinline__ void load(const void* p, long at, int c0, int c1, f32x4& x, f32x4& y) {
    if constexpr (BF16) {
      const bf16* q = static_cast<const bf16*>(p) + at;
      if constexpr (NEAR) {
        const bf16x8 z = *reinterpret_cast<const bf16x8*>(q + c0);
        x = __builtin_convertvector(__builtin_shufflevector(z, z, 0, 1, 2, 3), f32x4);
        y = __builtin_convertvector(__builtin_shufflevector(z, z, 4, 5, 6, 7), f32x4);
      } else {
        x = __builtin_convertvector(*reinterpret_cast<const bf16x4*>(q + c0), f32x4);
        y = __builtin_convertvector(*reinterpret_cast<const bf16x4*>(q + c1), f32x4);
      }
    } else {
      const float* q = static_cast<const float*>(p) + at;
      x = *reinterpret_cast<const f32x4u*>(q + c0);
      y = *reinterpret_cast<const f32x4u*>(q + c1);
    }
  }
  static __device__ __forceinline__ void store(void* p, long at, int c0, int c1, f32x4 x, f32x4 y) {
    if constexpr (BF16) {
      bf16* q = static_cast<bf16*>(p) + at;
      const bf16x4 u = to_bf16x4(x), v = to_bf16x4(y);
      if constexpr (NEAR) {
        put<PAST>(__builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7), q + c0);
      } else {
        put<PAST>(u, q + c0);
        put<PAST>(v, q + c1);
      }
    } else {
      float* q = static_cast<float*>(p) + at;
      put<PAST, f32x4u>(x, q + c0);
      put<PAST, f32x4u>(y, q + c1);
    }
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

// U neighbouring heads per thread, that share a row's angles. NEAR: the 8 values are neighbours (pairs are, or
// there is no rotation).
template <bool BF16, int DH, bool NEAR, int U, bool PAST>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRope a, FastDiv units) {
  constexpr int L = DH / 8;
  const int lane = threadIdx.x % L;
  const long base = (long)blockIdx.x * (kThreads / L), row0 = base / units.d;
  const uint32_t f = (uint32_t)(base - row0 * units.d) + threadIdx.x / L, over = units.quot(f);
  const long row = row0 + over;
  if (row >= a.n) return;
  const int unit = (int)(f - over * units.d);

  // this lane's channels c0 .. c0+3 and c1 .. c1+3, and its first pair
  int c0 = lane * 8, c1 = c0 + 4, pair = lane * 4;
  if constexpr (!NEAR) {
    const int half = a.rope_dim / 2;
    c0 = pair < half ? pair : pair + half;
    c1 = c0 + (pair < half ? half : (DH - a.rope_dim) / 2);
  }
  f32x4 x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = unit * U + u;
    x[u] = y[u] = (f32x4){};
    if (h < a.heads) Eight<BF16, NEAR, PAST>::load(a.q, row * a.q_stride + h * DH, c0, c1, x[u], y[u]);
    else if (h < a.heads + a.kv_heads) Eight<BF16, NEAR, PAST>::load(a.k, row * a.k_stride + (h - a.heads) * DH, c0, c1, x[u], y[u]);
  }
  // channels that are not turned are kept, not turned by 0: their pair may hold what is not finite
  bool turn = false;
  f32x4 cs[2] = {};
  if (pair < a.rope_dim / 2) {
    const long p = a.pos ? a.pos[row] : row;
    turn = p >= 0 && p < a.n_pos;
    if (turn) {
      const f32x4* t = reinterpret_cast<const f32x4*>(a.rope + p * a.rope_dim + pair * 2);
      cs[0] = t[0];
      cs[1] = t[1];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fmaf(x[u][j], x[u][j], fmaf(y[u][j], y[u][j], sum));
    sum = head_sum<L>(sum);
    float g = 1.f / sqrtf(sum * (1.f / DH) + a.eps);
    // squares past fp32, or all of them so small that bits are lost beside a smaller eps: in 64 bits
    const bool far = sum > 0x1p125f || (sum < 0x1p-90f && a.eps < 0x1p-80f);
    if (__any(far)) {
      double s = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) s += (double)x[u][j] * x[u][j] + (double)y[u][j] * y[u][j];
      s = 1.0 / sqrt(head_sum<L>(s) / DH + a.eps);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (far) x[u][j] = (float)(x[u][j] * s), y[u][j] = (float)(y[u][j] * s);
      }
      if (far) g = 1.f;
    }
    const int h = unit * U + u;
    if (h >= a.heads + a.kv_heads) continue;
    const bool is_q = h < a.heads;
    const void* weight = is_q ? a.q_weight : a.k_weight;
    f32x4 wx = {1.f, 1.f, 1.f, 1.f}, wy = wx;
    if (weight) Eight<BF16, NEAR, PAST>::load(weight, 0, c0, c1, wx, wy);
    const f32x4 p = x[u] * g * wx, q = y[u] * g * wy;
    f32x4 v = p, w = q;
    if (turn) {
      if constexpr (NEAR) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x2 r = rope_rotate((f32x2){cs[0][2 * j], cs[0][2 * j + 1]}, p[2 * j], p[2 * j + 1]);
          const f32x2 t = rope_rotate((f32x2){cs[1][2 * j], cs[1][2 * j + 1]}, q[2 * j], q[2 * j + 1]);
          v[2 * j] = r[0], v[2 * j + 1] = r[1], w[2 * j] = t[0], w[2 * j + 1] = t[1];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x2 r = rope_rotate((f32x2){cs[j >> 1][2 * (j & 1)], cs[j >> 1][2 * (j & 1) + 1]}, p[j], q[j]);
          v[j] = r[0], w[j] = r[1];
        }
      }
    }
    if (is_q) Eight<BF16, NEAR, PAST>::store(a.q_out, row * a.qo_stride + h * DH, c0, c1, v, w);
    else Eight<BF16, NEAR, PAST>::store(a.k_out, row * a.ko_stride + (h - a.heads) * DH, c0, c1, v, w);
  }
}

template <bool BF16, int DH, bool NEAR, int U, bool PAST>
hipError_t launch(const NormRope& a, hipStream_t s) {
  constexpr int per = kThreads / (DH / 8);
  const uint32_t units = (uint32_t)(a.heads + a.kv_heads + U - 1) / U;
  const long groups = ((long)a.n * units + per - 1) / per;
  hipLaunchKernelGGL((norm_rope_kernel<BF16, DH, NEAR, U, PAST>), dim3((unsigned)groups), dim3(kThreads), 0, s, a, FastDiv(units));
  return hipGetLastError();
}

template <bool BF16, int DH>
hipError_t launch_pairs(const NormRope& a, hipStream_t s) {
  // Two heads to a thread, in bf16, and stores past the caches where there are many: 8190 rows of 80 heads 72 us, 73 with one
  // head, 78 with that and ordinary stores, 91 with four (their registers); fp32 130 with two heads and 121 with one.
  const bool many = (long)a.n * (a.heads + a.kv_heads) * DH >= 1L << 22, near = a.interleaved || a.rope_dim == 0;
  constexpr int U = BF16 ? 2 : 1;
  if (many) return near ? launch<BF16, DH, true, U, true>(a, s) : launch<BF16, DH, false, U, true>(a, s);
  return near ? launch<BF16, DH, true, 1, false>(a, s) : launch<BF16, DH, false, 1, false>(a, s);
}

}  // namespace

hipError_t launch_norm_rope(const NormRope& a, bool bf16, int head_dim, hipStream_t s) {
  if (a.n <= 0 || a.heads + a.kv_heads <= 0) return hipSuccess;
  if (bf16) return head_dim == 64 ? launch_pairs<true, 64>(a, s) : launch_pairs<true, 128>(a, s);
  return head_dim == 64 ? launch_pairs<false, 64>(a, s) : launch_pairs<false, 128>(a, s);
}

}  // namespace hsa
