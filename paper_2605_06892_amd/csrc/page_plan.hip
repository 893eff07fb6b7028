// Pages and cache rows of the fresh tokens of many sequences, from their lengths alone.
//
// With f_s fresh tokens of sequence s (cut so that their sum is at most the capacity) and p_s rows
// before them, three exclusive sums say everything: where its tokens begin in the packed order
// (of f), how many rows it then has, and where its new pages begin in the free ring (of the pages
// that p_s + f_s rows need beyond those of p_s). Every workgroup forms the sums of all sequences,
// kChunk at a time, and writes what belongs to its own tokens: a token's sequence is found by a
// search in the sums, its page is an old entry of the table or the ring's, and the token
// that is the first of a new page writes it to the table. No workgroup waits for another.
// Writing is all there is to it: 8 bytes per token; up to some 10^5 tokens the launch bounds it.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;                   // sequences per thread
constexpr int kChunk = kThreads * kPer;   // sequences at a time
constexpr int kTile = 1024;               // tokens at a time

struct Lengths {
  int past, rows, have;  // rows before, all rows (at most the table's), pages before
};

// x + y, at most `most`: for terms of 0 to `most` < 2^30 an associative sum that cannot wrap
__device__ __forceinline__ int add_to(int x, int y, int most) { return min(x + y, most); }

// Exclusive sums of each thread's kPer values over the workgroup after `base`, at most `most`; returns the whole sum.
__device__ __forceinline__ int exclusive(int (&v)[kPer], int base, int most, int* waves) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int own = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) own = add_to(own, v[i], most);
  int sum = own;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(sum, o);
    if (lane >= o) sum = add_to(sum, y, most);
  }
  int before = __shfl_up(sum, 1);
  if (lane == 0) before = 0;
  __syncthreads();  // the last sums were read
  if (lane == kWave - 1) waves[wave] = sum;
  __syncthreads();
  int all = base;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w == wave) before = add_to(all, before, most);
    all = add_to(all, waves[w], most);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = v[i];
    v[i] = before;
    before = add_to(before, x, most);
  }
  return all;
}

struct Ring {
  int first, count;
  __device__ __forceinline__ explicit Ring(const PagePlan& a) {
    first = a.n_free > 0 ? (int)((unsigned)a.free_at[0] % (unsigned)a.n_free) : 0;
    count = min(max(a.free_at[1], 0), a.n_free);
  }
};

__global__ __launch_bounds__(kThreads) void page_plan_kernel(PagePlan a, FastDiv page, int* lens_out, int* next_out) {
  __shared__ int begins[kChunk + 1], pasts[kChunk], news[kChunk];  // first token, rows before, first new page
  __shared__ int waves[kThreads / kWave];
  const int most = a.n_tokens, rows_most = a.max_pages * a.page_size;
  const Ring ring(a);
  int tokens = 0, pages = 0;  // before this chunk
  for (long s0 = 0; s0 < a.n_seqs; s0 += kChunk) {
    const int n = (int)min((long)kChunk, a.n_seqs - s0);
    int at[kPer], fresh[kPer], past[kPer], need[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = threadIdx.x * kPer + i;
      fresh[i] = j < n ? min(max(a.fresh[s0 + j], 0), most) : 0;
      past[i] = j < n ? min(max(a.past[s0 + j], 0), rows_most) : 0;
      at[i] = fresh[i];
    }
    const int tokens_end = exclusive(at, tokens, most, waves);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = threadIdx.x * kPer + i;
      fresh[i] = add_to(at[i], fresh[i], most) - at[i];
      const int rows = min(past[i] + fresh[i], rows_most);
      need[i] = (int)(page.quot(rows + a.page_size - 1) - page.quot(past[i] + a.page_size - 1));
      if (blockIdx.x == 0 && j < n) {
        a.cu[s0 + j] = at[i];
        if (lens_out) lens_out[s0 + j] = rows;
      }
      begins[j] = at[i];
      pasts[j] = past[i];
    }
    const int pages_end = exclusive(need, pages, INT32_MAX / 2, waves);
#pragma unroll
    for (int i = 0; i < kPer; ++i) news[threadIdx.x * kPer + i] = need[i];
    if (threadIdx.x == 0) begins[kChunk] = tokens_end;
    __syncthreads();
    for (long t0 = ((long)(tokens / kTile - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x * (int)gridDim.x + (int)blockIdx.x) * kTile;
         t0 < tokens_end; t0 += (long)gridDim.x * kTile) {
      for (int t = max((int)t0, tokens) + threadIdx.x; t < min(t0 + kTile, (long)tokens_end); t += kThreads) {
        int lo = 0, hi = n;  // the last sequence that begins at t or before
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (begins[mid] <= t) lo = mid; else hi = mid;
        }
        const int pos = pasts[lo] + (t - begins[lo]);
        int slot = -1;
        if (pos < rows_most) {
          const int rank = (int)page.quot(pos), in = pos - rank * a.page_size;
          const int have = (int)page.quot(pasts[lo] + a.page_size - 1);
          int32_t* entry = a.page_table + (s0 + lo) * (long)a.max_pages + rank;
          int number;
          if (rank < have) {
            number = *entry;
          } else {
            const int j = news[lo] + rank - have;
            number = j < ring.count ? a.free_pages[ring.first + (long)j >= a.n_free ? ring.first + (long)j - a.n_free : ring.first + j] : -1;
            if (in == 0) *entry = number;
          }
          const long row = (long)number * a.page_size + in;
          slot = number < 0 || row > INT32_MAX ? -1 : (int)row;
        }
        a.pos[t] = pos;
        a.slots[t] = slot;
      }
    }
    __syncthreads();  // the sums were read
    tokens = tokens_end;
    pages = pages_end;
  }
  for (long t = tokens + (long)blockIdx.x * kThreads + threadIdx.x; t < a.n_tokens; t += (long)gridDim.x * kThreads) {
    a.pos[t] = -1;
    a.slots[t] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.cu[a.n_seqs] = tokens;
    if (next_out) {
      const int taken = min(pages, ring.count);
      const long next = (long)ring.first + taken;
      next_out[0] = (int)(next >= a.n_free && a.n_free > 0 ? next - a.n_free : next);
      next_out[1] = ring.count - taken;
      next_out[2] = pages - taken;
    }
  }
}

// What replaces its own input, after every workgroup above has read that: the lengths
// from the offsets, and the ring's state.
__global__ __launch_bounds__(kThreads) void page_plan_finish_kernel(PagePlan a, FastDiv page) {
  __shared__ int sums[kThreads / kWave];
  const int rows_most = a.max_pages * a.page_size;
  const Ring ring(a);
  int pages = 0;
  for (long s = threadIdx.x; s < a.n_seqs; s += kThreads) {
    const int past = min(max(a.past[s], 0), rows_most), rows = min(past + (a.cu[s + 1] - a.cu[s]), rows_most);
    if (a.kv_lens == a.past) a.kv_lens[s] = rows;
    pages += (int)(page.quot(rows + a.page_size - 1) - page.quot(past + a.page_size - 1));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) pages += __shfl_xor(pages, o);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = pages;
  __syncthreads();
  if (threadIdx.x > 0 || a.free_next != a.free_at) return;
  pages = 0;
  for (int w = 0; w < kThreads / kWave; ++w) pages += sums[w];
  const int taken = min(pages, ring.count);
  const long next = (long)ring.first + taken;
  a.free_next[0] = (int)(next >= a.n_free && a.n_free > 0 ? next - a.n_free : next);
  a.free_next[1] = ring.count - taken;
  a.free_next[2] = pages - taken;
}

}  // namespace

hipError_t launch_page_plan(const PagePlan& a, hipStream_t s) {
  const bool lens_here = a.kv_lens == a.past && a.n_seqs > 0, ring_here = a.free_next == a.free_at;
  const long tiles = ((long)a.n_tokens + kTile - 1) / kTile;
  const unsigned groups = (unsigned)(tiles < 1 ? 1 : tiles < 4L * compute_units() ? tiles : 4L * compute_units());
  const FastDiv page((uint32_t)a.page_size);
  hipLaunchKernelGGL(page_plan_kernel, dim3(groups), dim3(kThreads), 0, s, a, page, lens_here ? nullptr : a.kv_lens,
                     ring_here ? nullptr : a.free_next);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!lens_here && !ring_here)) return e;
  hipLaunchKernelGGL(page_plan_finish_kernel, dim3(1), dim3(kThreads), 0, s, a, page);
  return hipGetLastError();
}

}  // namespace hsa
