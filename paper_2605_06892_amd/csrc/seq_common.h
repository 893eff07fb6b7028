// What the kernels over several sequences share: e4m3 and e2m1 rows, divisions by
// sizes known on the host, and the launch arguments of their entry points.
#pragma once

#include "attention_util.h"

namespace hsa {

// Exponents of e4m3 cache rows. 2^e and 2^-e are normal numbers, the least code
// (2^-9) times 2^kExpMin still is one, and 448 * 2^kExpMax is finite.
constexpr int kExpMin = -117, kExpMax = 119;

// How rows are held: in their own type; e4m3 codes with an exponent per row and head;
// e2m1 codes, two to a byte, with an exponent per group of 32 values.
enum Held { kOwn, kE4M3, kE2M1 };
constexpr int kGroup = 32;

// Exponents of e2m1 groups. 2^e and 2^-e are normal numbers, so is the least code (1/2) times
// 2^kExp4Min, and 6 * 2^kExp4Max is finite. kExp4Nan marks a group that holds a
// value which is not finite: as the scale operand of the conversions from e2m1, 2^kExp4Nan (all
// exponent bits set) makes every code, 0 too, a NaN.
constexpr int kExp4Min = -125, kExp4Max = 125, kExp4Nan = -128;

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// 8 e2m1 codes of a word as bf16, times a power of two: exact
__device__ __forceinline__ bf16x8 widen4(unsigned c, float scale) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
  return (bf16x8){p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
}

// 8 fp32 values as three bf16 parts each, cut from the top: 8 + 8 + 8 bits, all that they have, but
// for what lies under bf16's least value, 2^-133. What is not finite is its first part alone.
__device__ __forceinline__ void cut3(const float (&x)[8], bf16x8 (&part)[3]) {
  unsigned h[8], m[8], l[8];
  float odd = 0.f;  // NaN if a value is not finite, for what is left of that then is
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    h[j] = __float_as_uint(x[j]);
    const float r = x[j] - __uint_as_float(h[j] & 0xffff0000u);
    m[j] = __float_as_uint(r);
    const float t = r - __uint_as_float(m[j] & 0xffff0000u);
    l[j] = __float_as_uint(t);
    odd += t;
  }
  if (__any(odd != odd)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned mag = h[j] & 0x7fffffffu;
      if (mag >= 0x7f800000u) m[j] = l[j] = 0;
      if (mag > 0x7f800000u) h[j] |= 0x00400000u;  // a NaN whose upper bits say infinity
    }
  }
  u32x4 p[3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {  // the upper halves of two
    p[0][j] = __builtin_amdgcn_perm(h[2 * j + 1], h[2 * j], 0x07060302);
    p[1][j] = __builtin_amdgcn_perm(m[2 * j + 1], m[2 * j], 0x07060302);
    p[2][j] = __builtin_amdgcn_perm(l[2 * j + 1], l[2 * j], 0x07060302);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) part[i] = __builtin_bit_cast(bf16x8, p[i]);
}

// x / d for 0 <= x < 2^31 by a multiplication: with s = ceil(log2 d) and m =
// floor(2^32 (2^s - d) / d) + 1 the quotient is (mulhi(x, m) + x) >> s.
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div), s(0) {
    while ((1ull << s) < div) ++s;
    m = (uint32_t)(((1ull << 32) * ((1ull << s) - div)) / div + 1);
  }
  __device__ __forceinline__ uint32_t quot(uint32_t x) const { return (__umulhi(x, m) + x) >> s; }
};

// Fresh rows in, or out of, a cache (cache.hip): rows of bf16 or fp32 values, and how the
// cache holds them.
struct CacheRows {
  bool bf16;
  Held held;
  const void *src_k, *src_v;    // rows read
  void *dst_k, *dst_v;          // rows written
  int8_t *k_exp, *v_exp;        // of codes
  long k_stride, v_stride;      // of the compact rows, in elements
  const int32_t* idx;
  int n;
  long n_rows;
  int kv_heads, head_dim;
};
hipError_t launch_cache_store(const CacheRows& c, hipStream_t s);
hipError_t launch_cache_load(const CacheRows& c, hipStream_t s);
// Rows of weights into e2m1 groups (cache.hip): d % 32 == 0, rows `stride` elements apart.
hipError_t launch_quantize_w4(const void* w, bool bf16, long n, int d, long stride, void* codes, int8_t* exps,
                              hipStream_t s);

// Attention of packed sequences (packed_attention.hip). Strides in elements.
struct PackedArgs {
  const void *q, *k, *v;
  long q_stride, k_stride, v_stride;
  const int32_t *cu_q, *cu_kv;
  int n_seqs, n_q, n_kv;
  int kv_heads, group;  // heads = kv_heads * group
  FastDiv by_group;
  float scale;
  int causal;
  void* o;
  float* lse;
};
hipError_t launch_packed_attention(const PackedArgs& a, bool bf16, int head_dim, hipStream_t s);

// One query per sequence over a paged cache (paged_attention.hip).
struct PagedArgs {
  const void* q;
  long q_stride;
  const void *k, *v;
  const int8_t *k_exp, *v_exp;
  const int32_t* page_table;
  const int32_t* kv_lens;
  int max_pages, n_seqs, n_pages, page_size;
  int kv_heads, group;
  float scale;
  void* o;
  float* lse;
  void* ws;
};
// Workspace bytes of a launch, 0 where no sequence can be split; more over e2m1 rows.
size_t paged_attention_bytes(int n_seqs, int kv_heads, int group, int head_dim, long max_len, bool e2m1);
hipError_t launch_paged_attention(const PagedArgs& a, bool bf16, Held held, int head_dim, hipStream_t s);

// Rows times weights in e2m1 groups (linear_w4.hip):
// y[m][o] = act(row_scale[m] sum_k x[m][k] w[o][k]) + residual[m][o].
struct LinearW4 {
  const void* x;          // [rows, d_in]
  const uint8_t* w;       // [d_out, d_in / 2]
  const int8_t* exps;     // [d_out, d_in / 32]
  int rows, d_in, d_out;
  const float* row_scale;
  const void* residual;   // of the output's type
  int gelu, out_f32;      // out_f32: bf16 rows, fp32 output
  void* y;
};
hipError_t launch_linear_w4(const LinearW4& a, bool bf16, hipStream_t s);

// Norms of query and key heads and their rotation (norm_rope.hip). Strides in elements.
struct NormRope {
  const void *q, *k;
  void *q_out, *k_out;
  long q_stride, k_stride, qo_stride, ko_stride;
  int n, heads, kv_heads;
  const void *q_weight, *k_weight;
  float eps;
  const float* rope;  // [n_pos, rope_dim / 2] (cos, sin)
  int rope_dim, interleaved;
  int64_t n_pos;
  const int32_t* pos;
};
hipError_t launch_norm_rope(const NormRope& a, bool bf16, int head_dim, hipStream_t s);

// Pages and cache rows of fresh tokens (page_plan.hip).
struct PagePlan {
  const int32_t *past, *fresh;
  int n_seqs, page_size, max_pages;
  int32_t* page_table;
  const int32_t* free_pages;
  int n_free;
  const int32_t* free_at;
  int n_tokens;
  int32_t *cu, *kv_lens, *pos, *slots, *free_next;
};
hipError_t launch_page_plan(const PagePlan& a, hipStream_t s);

}  // namespace hsa
