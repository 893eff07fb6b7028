// What the kernels over several sequences share: e4m3 rows, divisions by
// sizes known on the host, and the launch arguments of their entry points.
#pragma once

#include "attention_util.h"

namespace hsa {

// Exponents of e4m3 cache rows. 2^e and 2^-e are normal numbers, the least code
// (2^-9) times 2^kExpMin still is one, and 448 * 2^kExpMax is finite.
constexpr int kExpMin = -117, kExpMax = 119;

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

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

// Fresh rows in, or out of, a cache (cache.hip). `dtype` is the rows' type;
// e4m3: the cache holds codes and exponents, else rows of dtype.
struct CacheRows {
  bool bf16, e4m3;
  const void *src_k, *src_v;    // rows read
  void *dst_k, *dst_v;          // rows written
  int8_t *k_exp, *v_exp;        // e4m3
  long k_stride, v_stride;      // of the compact rows, in elements
  const int32_t* idx;
  int n;
  long n_rows;
  int kv_heads, head_dim;
};
hipError_t launch_cache_store(const CacheRows& c, hipStream_t s);
hipError_t launch_cache_load(const CacheRows& c, hipStream_t s);

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
// Workspace bytes of a launch, 0 where no sequence can be split.
size_t paged_attention_bytes(int n_seqs, int kv_heads, int group, int head_dim, long max_len);
hipError_t launch_paged_attention(const PagedArgs& a, bool bf16, bool e4m3, int head_dim, hipStream_t s);

}  // namespace hsa
