// C ABI entry points of the calls over several sequences: host-side argument
// checks, then kernel launches. See include/hsa_step.h for their contract.
#include "api_util.h"
#include "seq_common.h"

using namespace hsa_api;

namespace {

constexpr int64_t kMaxStride = int64_t(1) << 22;  // elements between rows
constexpr int64_t kMaxKeys = int64_t(1) << 30;    // keys of a sequence, so that a position plus a block fits an int
constexpr int64_t kMaxLaunch = int64_t(1) << 32;  // threads of one launch

// Bytes from the first to the end of the last of n rows `stride` elements apart.
size_t span(int64_t n, int64_t stride, int64_t width, size_t es) {
  return n > 0 ? ((size_t)(n - 1) * (size_t)stride + (size_t)width) * es : 0;
}

// Rows of a strided input: their stride and alignment (bf16 16 bytes, fp32 4).
bool rows_ok(const void* p, int64_t n, int64_t stride, int64_t width, size_t es) {
  if (stride < width || stride > kMaxStride || !fits(n, stride, es)) return false;
  return es == 2 ? aligned(p, 16) && stride % 8 == 0 : aligned(p, 4);
}

bool heads_ok(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  return heads > 0 && kv_heads > 0 && heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128) &&
         (int64_t)heads * head_dim <= kMaxStride;
}

// the kernels take scale * log2(e) in fp32
bool scale_ok(float scale) { return scale > 0.f && scale <= 0x1p127f; }

struct Range {
  const void* p;
  size_t n;
};

// True if the first `outs` ranges overlap each other or any later range.
template <int N>
bool any_overlap(const Range (&r)[N], int outs) {
  for (int i = 0; i < outs; ++i)
    for (int j = i + 1; j < N; ++j)
      if (overlaps(r[i].p, r[i].n, r[j].p, r[j].n)) return true;
  return false;
}

// The cache's element size; 0 unless cache_dtype is dtype or e4m3.
size_t cache_elem(int dtype, int cache_dtype) {
  if (cache_dtype == HSA_STEP_E4M3) return 1;
  return cache_dtype == dtype ? elem_size(dtype) : 0;
}

// Checks of hsa_cache_store and hsa_cache_load that do not depend on the direction.
int check_cache(int dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                const int32_t* idx, int32_t n, int64_t n_rows, int32_t kv_heads, int32_t head_dim,
                int cache_dtype, const void* k_cache, const void* v_cache, const int8_t* k_exp,
                const int8_t* v_exp) {
  const size_t es = elem_size(dtype), ce = cache_elem(dtype, cache_dtype);
  if (!es || !ce) return HSA_STEP_ERR_DTYPE;
  if (n < 0 || n_rows < 0 || n_rows > kMaxRows || !heads_ok(kv_heads, kv_heads, head_dim)) return HSA_STEP_ERR_SHAPE;
  const int64_t d = (int64_t)kv_heads * head_dim;
  // one launch: fewer than 2^32 threads of 8 values
  if (!fits(n_rows, d, ce) || (int64_t)n * d >= kMaxLaunch * 4) return HSA_STEP_ERR_SHAPE;
  if (n == 0) return HSA_STEP_OK;
  if (!k || !v || !idx || (n_rows > 0 && (!k_cache || !v_cache))) return HSA_STEP_ERR_NULL;
  const bool exps = cache_dtype == HSA_STEP_E4M3;
  if (exps && n_rows > 0 && (!k_exp || !v_exp)) return HSA_STEP_ERR_NULL;
  const size_t ca = ce == 4 ? 4 : 16;
  if (!rows_ok(k, n, k_stride, d, es) || !rows_ok(v, n, v_stride, d, es) || !aligned(idx, 4) ||
      !aligned(k_cache, ca) || !aligned(v_cache, ca))
    return HSA_STEP_ERR_SHAPE;
  return HSA_STEP_OK;
}

}  // namespace

HSA_API int hsa_cache_store(int dtype, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const int32_t* idx, int32_t n, int64_t n_rows,
                            int32_t kv_heads, int32_t head_dim, int cache_dtype, void* k_cache,
                            void* v_cache, int8_t* k_exp, int8_t* v_exp, hipStream_t stream) {
  const int st = check_cache(dtype, k, k_stride, v, v_stride, idx, n, n_rows, kv_heads, head_dim,
                             cache_dtype, k_cache, v_cache, k_exp, v_exp);
  if (st != HSA_STEP_OK || n == 0) return st;
  const int64_t d = (int64_t)kv_heads * head_dim;
  const bool e4m3 = cache_dtype == HSA_STEP_E4M3;
  const size_t cb = (size_t)n_rows * d * cache_elem(dtype, cache_dtype);
  const size_t eb = e4m3 ? (size_t)n_rows * kv_heads : 0;
  const size_t es = elem_size(dtype);
  const Range r[] = {{k_cache, cb}, {v_cache, cb}, {k_exp, eb}, {v_exp, eb}, {k, span(n, k_stride, d, es)},
                     {v, span(n, v_stride, d, es)}, {idx, (size_t)n * 4}};
  if (any_overlap(r, 4)) return HSA_STEP_ERR_ALIAS;
  if (n_rows == 0) return HSA_STEP_OK;
  hsa::CacheRows c{};
  c.bf16 = dtype == HSA_STEP_BF16;
  c.e4m3 = e4m3;
  c.src_k = k;
  c.src_v = v;
  c.dst_k = k_cache;
  c.dst_v = v_cache;
  c.k_exp = k_exp;
  c.v_exp = v_exp;
  c.k_stride = k_stride;
  c.v_stride = v_stride;
  c.idx = idx;
  c.n = n;
  c.n_rows = n_rows;
  c.kv_heads = kv_heads;
  c.head_dim = head_dim;
  return launch_status(hsa::launch_cache_store(c, stream));
}

HSA_API int hsa_cache_load(int cache_dtype, const void* k_cache, const void* v_cache,
                           const int8_t* k_exp, const int8_t* v_exp, const int32_t* idx, int32_t n,
                           int64_t n_rows, int32_t kv_heads, int32_t head_dim, int dtype, void* k,
                           int64_t k_stride, void* v, int64_t v_stride, hipStream_t stream) {
  const int st = check_cache(dtype, k, k_stride, v, v_stride, idx, n, n_rows, kv_heads, head_dim,
                             cache_dtype, k_cache, v_cache, k_exp, v_exp);
  if (st != HSA_STEP_OK || n == 0) return st;
  const int64_t d = (int64_t)kv_heads * head_dim;
  const bool e4m3 = cache_dtype == HSA_STEP_E4M3;
  const size_t cb = (size_t)n_rows * d * cache_elem(dtype, cache_dtype);
  const size_t eb = e4m3 ? (size_t)n_rows * kv_heads : 0;
  const size_t es = elem_size(dtype);
  const Range r[] = {{k, span(n, k_stride, d, es)}, {v, span(n, v_stride, d, es)}, {k_cache, cb}, {v_cache, cb},
                     {k_exp, eb}, {v_exp, eb}, {idx, (size_t)n * 4}};
  if (any_overlap(r, 2)) return HSA_STEP_ERR_ALIAS;
  hsa::CacheRows c{};
  c.bf16 = dtype == HSA_STEP_BF16;
  c.e4m3 = e4m3;
  c.src_k = k_cache;
  c.src_v = v_cache;
  c.dst_k = k;
  c.dst_v = v;
  c.k_exp = const_cast<int8_t*>(k_exp);
  c.v_exp = const_cast<int8_t*>(v_exp);
  c.k_stride = k_stride;
  c.v_stride = v_stride;
  c.idx = idx;
  c.n = n;
  c.n_rows = n_rows;
  c.kv_heads = kv_heads;
  c.head_dim = head_dim;
  return launch_status(hsa::launch_cache_load(c, stream));
}

HSA_API int hsa_packed_attention(int dtype, const void* q, int64_t q_stride, const void* k,
                                 int64_t k_stride, const void* v, int64_t v_stride,
                                 const int32_t* cu_q, const int32_t* cu_kv, int32_t n_seqs,
                                 int64_t n_q, int64_t n_kv, int32_t heads, int32_t kv_heads,
                                 int32_t head_dim, float scale, int32_t causal, void* o, float* lse,
                                 hipStream_t stream) {
  const size_t es = elem_size(dtype);
  if (!es) return HSA_STEP_ERR_DTYPE;
  if (!heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || n_seqs == INT32_MAX || n_q < 0 || n_kv < 0 ||
      n_q > kMaxRows / heads || n_kv > kMaxKeys || !scale_ok(scale))
    return HSA_STEP_ERR_SHAPE;
  // one launch: fewer than 2^32 threads, 512 per 16 rows or item
  if (n_q * heads / 16 + ((int64_t)n_seqs + 8) * kv_heads >= kMaxLaunch / 512) return HSA_STEP_ERR_SHAPE;
  if (n_q == 0 || n_seqs == 0) return HSA_STEP_OK;
  if (!q || !cu_q || !cu_kv || !o || (n_kv > 0 && (!k || !v))) return HSA_STEP_ERR_NULL;
  const int64_t d = (int64_t)heads * head_dim, dk = (int64_t)kv_heads * head_dim;
  if (!rows_ok(q, n_q, q_stride, d, es) || (n_kv > 0 && (!rows_ok(k, n_kv, k_stride, dk, es) || !rows_ok(v, n_kv, v_stride, dk, es))) ||
      !aligned(o, es == 2 ? 16 : 4) || !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(cu_kv, 4))
    return HSA_STEP_ERR_SHAPE;
  const size_t cub = ((size_t)n_seqs + 1) * 4;
  const Range r[] = {{o, (size_t)n_q * d * es}, {lse, lse ? (size_t)n_q * heads * 4 : 0}, {q, span(n_q, q_stride, d, es)},
                     {k, span(n_kv, k_stride, dk, es)}, {v, span(n_kv, v_stride, dk, es)}, {cu_q, cub}, {cu_kv, cub}};
  if (any_overlap(r, 2)) return HSA_STEP_ERR_ALIAS;
  hsa::PackedArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.cu_q = cu_q;
  a.cu_kv = cu_kv;
  a.n_seqs = n_seqs;
  a.n_q = (int)n_q;
  a.n_kv = (int)n_kv;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.by_group = hsa::FastDiv((uint32_t)a.group);
  a.scale = scale;
  a.causal = causal != 0;
  a.o = o;
  a.lse = lse;
  return launch_status(hsa::launch_packed_attention(a, dtype == HSA_STEP_BF16, head_dim, stream));
}

HSA_API size_t hsa_paged_attention_workspace_bytes(int dtype, int32_t n_seqs, int32_t heads,
                                                   int32_t kv_heads, int32_t head_dim,
                                                   int64_t max_len) {
  if (!elem_size(dtype) || !heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || max_len < 0 ||
      max_len > kMaxKeys || n_seqs > kMaxRows / heads)
    return 0;
  return hsa::paged_attention_bytes(n_seqs, kv_heads, heads / kv_heads, head_dim, max_len);
}

HSA_API int hsa_paged_attention(int dtype, const void* q, int64_t q_stride, int cache_dtype,
                                const void* k_cache, const void* v_cache, const int8_t* k_exp,
                                const int8_t* v_exp, const int32_t* page_table, int32_t max_pages,
                                const int32_t* kv_lens, int32_t n_seqs, int32_t n_pages,
                                int32_t page_size, int32_t heads, int32_t kv_heads,
                                int32_t head_dim, float scale, void* o, float* lse,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const size_t es = elem_size(dtype), ce = cache_elem(dtype, cache_dtype);
  if (!es || !ce) return HSA_STEP_ERR_DTYPE;
  if (!heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || n_seqs > kMaxRows / heads || n_pages < 0 ||
      max_pages < 0 || page_size < 1 || (int64_t)n_pages * page_size > kMaxRows ||
      (int64_t)max_pages * page_size > kMaxKeys || !scale_ok(scale))
    return HSA_STEP_ERR_SHAPE;
  const int64_t d = (int64_t)heads * head_dim, dk = (int64_t)kv_heads * head_dim;
  const int64_t n_rows = (int64_t)n_pages * page_size;
  if (!fits(n_rows, dk, ce) || !fits(n_seqs, max_pages, 4) || (int64_t)n_seqs * heads >= kMaxLaunch / 512)
    return HSA_STEP_ERR_SHAPE;
  if (n_seqs == 0) return HSA_STEP_OK;
  const bool e4m3 = cache_dtype == HSA_STEP_E4M3;
  if (!q || !kv_lens || !o || (max_pages > 0 && !page_table) || (n_rows > 0 && (!k_cache || !v_cache)) ||
      (e4m3 && n_rows > 0 && (!k_exp || !v_exp)))
    return HSA_STEP_ERR_NULL;
  const size_t ca = ce == 4 ? 4 : 16;
  if (!rows_ok(q, n_seqs, q_stride, d, es) || !aligned(k_cache, ca) || !aligned(v_cache, ca) ||
      !aligned(o, es == 2 ? 16 : 4) || !aligned(lse, 4) || !aligned(page_table, 4) || !aligned(kv_lens, 4))
    return HSA_STEP_ERR_SHAPE;
  const size_t need = hsa_paged_attention_workspace_bytes(dtype, n_seqs, heads, kv_heads, head_dim,
                                                          (int64_t)max_pages * page_size);
  if (need && (!workspace || workspace_bytes < need)) return HSA_STEP_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return HSA_STEP_ERR_SHAPE;
  const size_t cb = (size_t)n_rows * dk * ce, eb = e4m3 ? (size_t)n_rows * kv_heads : 0;
  const Range r[] = {{o, (size_t)n_seqs * d * es}, {lse, lse ? (size_t)n_seqs * heads * 4 : 0}, {workspace, need},
                     {q, span(n_seqs, q_stride, d, es)}, {k_cache, cb}, {v_cache, cb}, {k_exp, eb}, {v_exp, eb},
                     {page_table, (size_t)n_seqs * max_pages * 4}, {kv_lens, (size_t)n_seqs * 4}};
  if (any_overlap(r, 3)) return HSA_STEP_ERR_ALIAS;
  hsa::PagedArgs a{};
  a.q = q;
  a.q_stride = q_stride;
  a.k = k_cache;
  a.v = v_cache;
  a.k_exp = k_exp;
  a.v_exp = v_exp;
  a.page_table = page_table;
  a.kv_lens = kv_lens;
  a.max_pages = max_pages;
  a.n_seqs = n_seqs;
  a.n_pages = n_pages;
  a.page_size = page_size;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.scale = scale;
  a.o = o;
  a.lse = lse;
  a.ws = workspace;
  return launch_status(hsa::launch_paged_attention(a, dtype == HSA_STEP_BF16, e4m3, head_dim, stream));
}
