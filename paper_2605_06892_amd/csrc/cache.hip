// Cache rows in 8 bits: written by row index as they are quantized, and read
// back. Both are streams: 8 values per thread and tensor, 16 bytes of bf16.
//
//   store  amax over a row's head (head_dim / 8 neighbouring lanes, three or four DPP
//          steps), e = the least exponent with amax <= 448 * 2^e, codes =
//          e4m3(x * 2^-e). The magnitudes are compared as integers (for finite
//          values the same order), so one packed maximum serves two bf16 values, and
//          whatever is not finite is found by the same comparison.
//   load   code * 2^e, exact in bf16 and fp32.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}

// maximum over the DH/8 lanes (8 or 16, aligned) that hold one head of a row
template <int DH>
__device__ __forceinline__ unsigned head_max(unsigned x) {
  x = max(x, dpp<0xB1>(x));   // lane ^ 1
  x = max(x, dpp<0x4E>(x));   // lane ^ 2
  x = max(x, dpp<0x141>(x));  // mirrored in 8
  if (DH == 128) x = max(x, dpp<0x140>(x));  // mirrored in 16
  return x;
}

// 8 values of one row, as they are held
template <bool BF16>
struct Vals;
template <>
struct Vals<true> {
  u32x4 x;
  __device__ __forceinline__ void load(const void* p, long i) {
    x = *reinterpret_cast<const u32x4*>(static_cast<const bf16*>(p) + i);
  }
  __device__ __forceinline__ void store(void* p, long i) const {
    *reinterpret_cast<u32x4*>(static_cast<bf16*>(p) + i) = x;
  }
  __device__ __forceinline__ void zero() { x = (u32x4){}; }
  __device__ __forceinline__ float at(int j) const {
    return __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16);
  }
  // greatest magnitude as the bits of an fp32 value (whose low half is 0)
  __device__ __forceinline__ unsigned top() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[j] & 0x7fff7fffu));
    return (unsigned)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ void set(int j, float lo, float hi) {  // values 2j and 2j+1, exact in bf16
    x[j] = (__float_as_uint(lo) >> 16) | (__float_as_uint(hi) & 0xffff0000u);
  }
};
template <>
struct Vals<false> {
  f32x4 x[2];
  __device__ __forceinline__ void load(const void* p, long i) {
    const float* f = static_cast<const float*>(p) + i;
    x[0] = *reinterpret_cast<const f32x4u*>(f);
    x[1] = *reinterpret_cast<const f32x4u*>(f + 4);
  }
  __device__ __forceinline__ void store(void* p, long i) const {
    float* f = static_cast<float*>(p) + i;
    *reinterpret_cast<f32x4u*>(f) = x[0];
    *reinterpret_cast<f32x4u*>(f + 4) = x[1];
  }
  __device__ __forceinline__ void zero() { x[0] = x[1] = (f32x4){}; }
  __device__ __forceinline__ float at(int j) const { return x[j >> 2][j & 3]; }
  __device__ __forceinline__ unsigned top() const {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(at(j)) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void set(int j, float lo, float hi) {
    x[j >> 1][2 * (j & 1)] = lo;
    x[j >> 1][2 * (j & 1) + 1] = hi;
  }
};

// codes of 8 values, and their head's exponent (the same in all its lanes)
template <bool BF16, int DH>
__device__ __forceinline__ u32x2 quantize(const Vals<BF16>& v, int& e) {
  constexpr unsigned kInf = 0x7f800000u, kSat = 0x7f600000u;  // infinity; 448 * 2^kExpMax
  unsigned m = head_max<DH>(v.top());
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = v.at(j);
  unsigned odd = 0;  // values that are not finite
  const bool wide = m > kSat;
  if (__any(wide)) {
    unsigned f = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned a = __float_as_uint(y[j]) & 0x7fffffffu;
      if (a >= kInf) odd |= 1u << j; else f = max(f, a);
    }
    m = head_max<DH>(f);
  }
  // 448 = 1.75 * 2^8: the next exponent up where the fraction is above 1.75
  e = min(max((int)((m + 0x1fffffu) >> 23) - 8 - 127, kExpMin), kExpMax);
  const float inv = pow2(-e);
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] *= inv;
  if (__any(wide)) {
#pragma unroll
    for (int j = 0; j < 8; ++j)  // the NaN code from a NaN, whatever its head's exponent
      y[j] = odd >> j & 1 ? __uint_as_float(0x7fc00000u) : fminf(fmaxf(y[j], -448.f), 448.f);
  }
  u32x2 c;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j], y[4 * j + 1], 0, false);
    c[j] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j + 2], y[4 * j + 3], w, true);
  }
  return c;
}

template <bool BF16>
__device__ __forceinline__ Vals<BF16> values(u32x2 c, int e) {
  const float s = pow2(e);
  Vals<BF16> v;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[j], false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[j], true);
    v.set(2 * j, a[0] * s, a[1] * s);
    v.set(2 * j + 1, b[0] * s, b[1] * s);
  }
  return v;
}

// Row and chunk of this thread's unit i of its workgroup: units are the 8-value
// chunks of the n rows in order, kThreads * U to a workgroup.
struct Units {
  long row0;
  uint32_t rest;
  template <int U>
  static __device__ __forceinline__ Units of_group(uint32_t cpr) {
    const long base = (long)blockIdx.x * (kThreads * U);
    Units u;
    u.row0 = base / cpr;
    u.rest = (uint32_t)(base - u.row0 * cpr);
    return u;
  }
};

template <bool BF16, int DH, bool E4M3, int U>
__global__ __launch_bounds__(kThreads) void store_kernel(CacheRows c, FastDiv cpr) {
  const Units g = Units::of_group<U>(cpr.d);
  Vals<BF16> kx[U], vx[U];
  long dst[U];
  int col[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t f = g.rest + i * kThreads + threadIdx.x, q = cpr.quot(f);
    const long j = g.row0 + q;
    col[i] = (int)(f - q * cpr.d) * 8;
    dst[i] = -1;
    kx[i].zero();
    vx[i].zero();
    if (j < c.n) {
      kx[i].load(c.src_k, j * c.k_stride + col[i]);
      vx[i].load(c.src_v, j * c.v_stride + col[i]);
      const int t = c.idx[j];
      if (t >= 0 && t < c.n_rows) dst[i] = t;
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const long at = dst[i] * (long)(cpr.d * 8) + col[i];
    if constexpr (E4M3) {
      int ke, ve;
      const u32x2 kc = quantize<BF16, DH>(kx[i], ke), vc = quantize<BF16, DH>(vx[i], ve);
      if (dst[i] < 0) continue;
      *reinterpret_cast<u32x2*>(static_cast<char*>(c.dst_k) + at) = kc;
      *reinterpret_cast<u32x2*>(static_cast<char*>(c.dst_v) + at) = vc;
      if (col[i] % DH == 0) {
        const long h = dst[i] * c.kv_heads + col[i] / DH;
        c.k_exp[h] = (int8_t)ke;
        c.v_exp[h] = (int8_t)ve;
      }
    } else {
      if (dst[i] < 0) continue;
      kx[i].store(c.dst_k, at);
      vx[i].store(c.dst_v, at);
    }
  }
}

template <bool BF16, int DH, bool E4M3, int U>
__global__ __launch_bounds__(kThreads) void load_kernel(CacheRows c, FastDiv cpr) {
  const Units g = Units::of_group<U>(cpr.d);
  Vals<BF16> kx[U], vx[U];
  u32x2 kc[U], vc[U];
  int ke[U], ve[U], col[U];
  long row[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t f = g.rest + i * kThreads + threadIdx.x, q = cpr.quot(f);
    row[i] = g.row0 + q;
    col[i] = (int)(f - q * cpr.d) * 8;
    kx[i].zero();
    vx[i].zero();
    kc[i] = vc[i] = (u32x2){};
    ke[i] = ve[i] = 0;
    if (row[i] < c.n) {
      const int t = c.idx[row[i]];
      if (t >= 0 && t < c.n_rows) {
        const long at = (long)t * (long)(cpr.d * 8) + col[i];
        if constexpr (E4M3) {
          kc[i] = *reinterpret_cast<const u32x2*>(static_cast<const char*>(c.src_k) + at);
          vc[i] = *reinterpret_cast<const u32x2*>(static_cast<const char*>(c.src_v) + at);
          ke[i] = c.k_exp[(long)t * c.kv_heads + col[i] / DH];
          ve[i] = c.v_exp[(long)t * c.kv_heads + col[i] / DH];
        } else {
          kx[i].load(c.src_k, at);
          vx[i].load(c.src_v, at);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (row[i] >= c.n) continue;
    if constexpr (E4M3) {
      kx[i] = values<BF16>(kc[i], ke[i]);
      vx[i] = values<BF16>(vc[i], ve[i]);
    }
    kx[i].store(c.dst_k, row[i] * c.k_stride + col[i]);
    vx[i].store(c.dst_v, row[i] * c.v_stride + col[i]);
  }
}

template <bool STORE, bool BF16, int DH, bool E4M3>
hipError_t launch(const CacheRows& c, hipStream_t s) {
  constexpr int U = 1;
  const uint32_t cpr = (uint32_t)c.kv_heads * (DH / 8);
  const long groups = ((long)c.n * cpr + kThreads * U - 1) / (kThreads * U);
  if constexpr (STORE)
    hipLaunchKernelGGL((store_kernel<BF16, DH, E4M3, U>), dim3((unsigned)groups), dim3(kThreads), 0, s, c, FastDiv(cpr));
  else
    hipLaunchKernelGGL((load_kernel<BF16, DH, E4M3, U>), dim3((unsigned)groups), dim3(kThreads), 0, s, c, FastDiv(cpr));
  return hipGetLastError();
}

template <bool STORE, bool BF16, int DH>
hipError_t launch_held(const CacheRows& c, hipStream_t s) {
  return c.e4m3 ? launch<STORE, BF16, DH, true>(c, s) : launch<STORE, BF16, DH, false>(c, s);
}

template <bool STORE>
hipError_t launch_any(const CacheRows& c, hipStream_t s) {
  if (c.n <= 0) return hipSuccess;
  if (c.bf16) return c.head_dim == 64 ? launch_held<STORE, true, 64>(c, s) : launch_held<STORE, true, 128>(c, s);
  return c.head_dim == 64 ? launch_held<STORE, false, 64>(c, s) : launch_held<STORE, false, 128>(c, s);
}

}  // namespace

hipError_t launch_cache_store(const CacheRows& c, hipStream_t s) { return launch_any<true>(c, s); }
hipError_t launch_cache_load(const CacheRows& c, hipStream_t s) { return launch_any<false>(c, s); }

}  // namespace hsa
