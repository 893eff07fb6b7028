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

// What is read is read once and not kept in the caches: 8190 rows of 40 heads stored in
// 44 us against 51, 32760 rows of 12 heads loaded in 56 against 60. Values that are read
// back pass them by too (53); rows just stored stay, the next call may want them
// (and past the caches it takes 48).
template <class T>
__device__ __forceinline__ T get(const void* p) {
  return __builtin_nontemporal_load(static_cast<const T*>(p));
}
template <bool KEEP, class T>
__device__ __forceinline__ void put(T x, void* p) {
  if constexpr (KEEP) *static_cast<T*>(p) = x;
  else __builtin_nontemporal_store(x, static_cast<T*>(p));
}

// 8 values of one row, as they are held
template <bool BF16>
struct Vals;
template <>
struct Vals<true> {
  u32x4 x;
  __device__ __forceinline__ void load(const void* p, long i) {
    x = get<u32x4>(static_cast<const bf16*>(p) + i);
  }
  template <bool KEEP>
  __device__ __forceinline__ void store(void* p, long i) const {
    put<KEEP>(x, static_cast<bf16*>(p) + i);
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
    x[0] = get<f32x4u>(f);
    x[1] = get<f32x4u>(f + 4);
  }
  template <bool KEEP>
  __device__ __forceinline__ void store(void* p, long i) const {
    float* f = static_cast<float*>(p) + i;
    put<KEEP, f32x4u>(x[0], f);
    put<KEEP, f32x4u>(x[1], f + 4);
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

// Row and column (of the row's values) of this thread's 8 values: the chunks of the
// n rows in order, kThreads to a workgroup. One chunk of each tensor per
// thread: two took 3% longer at 8190 rows of 40 heads, four 10%.
struct Place {
  long row;
  int col;
  __device__ __forceinline__ explicit Place(FastDiv chunks) {
    const long base = (long)blockIdx.x * kThreads, row0 = base / chunks.d;
    const uint32_t f = (uint32_t)(base - row0 * chunks.d) + threadIdx.x, q = chunks.quot(f);
    row = row0 + q;
    col = (int)(f - q * chunks.d) * 8;
  }
};

template <bool BF16, int DH, bool E4M3>
__global__ __launch_bounds__(kThreads) void store_kernel(CacheRows c, FastDiv chunks) {
  const Place p(chunks);
  Vals<BF16> kx, vx;
  kx.zero();
  vx.zero();
  long dst = -1;
  if (p.row < c.n) {
    kx.load(c.src_k, p.row * c.k_stride + p.col);
    vx.load(c.src_v, p.row * c.v_stride + p.col);
    const int t = c.idx[p.row];
    if (t >= 0 && t < c.n_rows) dst = t;
  }
  const long at = dst * (long)(chunks.d * 8) + p.col;
  if constexpr (E4M3) {
    int ke, ve;
    const u32x2 kc = quantize<BF16, DH>(kx, ke), vc = quantize<BF16, DH>(vx, ve);
    if (dst < 0) return;
    put<true>(kc, static_cast<char*>(c.dst_k) + at);
    put<true>(vc, static_cast<char*>(c.dst_v) + at);
    if (p.col % DH == 0) {
      const long h = dst * c.kv_heads + p.col / DH;
      c.k_exp[h] = (int8_t)ke;
      c.v_exp[h] = (int8_t)ve;
    }
  } else {
    if (dst < 0) return;
    kx.template store<true>(c.dst_k, at);
    vx.template store<true>(c.dst_v, at);
  }
}

template <bool BF16, int DH, bool E4M3>
__global__ __launch_bounds__(kThreads) void load_kernel(CacheRows c, FastDiv chunks) {
  const Place p(chunks);
  if (p.row >= c.n) return;
  Vals<BF16> kx, vx;
  kx.zero();
  vx.zero();
  const int t = c.idx[p.row];
  if (t >= 0 && t < c.n_rows) {
    const long at = (long)t * (long)(chunks.d * 8) + p.col;
    if constexpr (E4M3) {
      const u32x2 kc = get<u32x2>(static_cast<const char*>(c.src_k) + at);
      const u32x2 vc = get<u32x2>(static_cast<const char*>(c.src_v) + at);
      const long h = (long)t * c.kv_heads + p.col / DH;
      const int ke = c.k_exp[h], ve = c.v_exp[h];
      kx = values<BF16>(kc, ke);
      vx = values<BF16>(vc, ve);
    } else {
      kx.load(c.src_k, at);
      vx.load(c.src_v, at);
    }
  }
  kx.template store<false>(c.dst_k, p.row * c.k_stride + p.col);
  vx.template store<false>(c.dst_v, p.row * c.v_stride + p.col);
}

template <bool STORE, bool BF16, int DH, bool E4M3>
hipError_t launch(const CacheRows& c, hipStream_t s) {
  const uint32_t chunks = (uint32_t)c.kv_heads * (DH / 8);  // of a row
  const long groups = ((long)c.n * chunks + kThreads - 1) / kThreads;
  if constexpr (STORE)
    hipLaunchKernelGGL((store_kernel<BF16, DH, E4M3>), dim3((unsigned)groups), dim3(kThreads), 0, s, c, FastDiv(chunks));
  else
    hipLaunchKernelGGL((load_kernel<BF16, DH, E4M3>), dim3((unsigned)groups), dim3(kThreads), 0, s, c, FastDiv(chunks));
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
