// Pages and cache rows of the fresh tokens of many sequences, from their lengths alone.
//
// With f_s fresh tokens of sequence s (cut so that their sum is at most the capacity) and p_s rows
// before them, three exclusive sums say everything: where its tokens begin in the packed order
// (of f), how many rows it then has, and where its new pages begin in the free ring (of the pages
// that p_s + f_s rows need beyond those of p_s). Every workgroup forms the sums of all sequences,
// kChunk at a time, and writes what belongs to its own tokens: a token's sequence is found by a
// search in the sums, its page is an old entry of the table or the ring's, and the token
// that is the first of a new page writes it to the table. No workgroup waits for another.
// Writing is all there is to it, 8 bytes per token; what takes the time is a chain of reads: lengths, the sums and the
// search in LDS, a page's number. A thousand prompts of 264 thousand tokens: 6.5 us with a token per thread, 9.2 with
// four in turn, 8 with four at once; 48 sequences of one token 4.6-5.3.
#include "seq_common.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;                   // sequences per thread
constexpr int kChunk = kThreads * kPer;   // sequences at a time
constexpr int kTile = kThreads;           // tokens at a time
typedef int i32x4u __attribute__((ext_vector_type(4), aligned(4)));

struct Lengths {
  int past, rows, have;  // rows before, all rows (at most the table's), pages before
};

// x + y, at most `most`: for terms of 0 to `most` < 2^30 an associative sum that cannot wrap
__device__ __forceinline__ int add_to(int x, int y, int most) { return min(x + y, most); }

// x of the lane that CTRL says, 0 where there is none and in the rows of 16 that ROWS leaves out
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true);
}

// Exclusive sums of each thread's kPer values over the workgroup after `base`, at most `most`; returns the whole sum.
__device__ __forceinline__ int exclusive(int (&v)[kPer], int base, int most, int* waves) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int own = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) own = add_to(own, v[i], most);
  // over 16 lanes, then the last of 16 to the next 16, of 32 to the next 32
  int sum = own;
  sum = add_to(sum, from_lane<0x111, 0xf>(sum), most);
  sum = add_to(sum, from_lane<0x112, 0xf>(sum), most);
  sum = add_to(sum, from_lane<0x114, 0xf>(sum), most);
  sum = add_to(sum, from_lane<0x118, 0xf>(sum), most);
  sum = add_to(sum, from_lane<0x142, 0xa>(sum), most);
  sum = add_to(sum, from_lane<0x143, 0xc>(sum), most);
  int before = from_lane<0x138, 0xf>(sum);  // the lane before
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
  __shared__ int begins[kChunk], pasts[kChunk], news[kChunk];  // first token, rows before, first new page
  __shared__ int waves[kThreads / kWave];
  const int most = a.n_tokens, rows_most = a.max_pages * a.page_size;
  const Ring ring(a);
  int tokens = 0, pages = 0;  // before this chunk
  for (long s0 = 0; s0 < a.n_seqs; s0 += kChunk) {
    const int n = (int)min((long)kChunk, a.n_seqs - s0);
    int at[kPer], fresh[kPer], past[kPer], need[kPer];
    const int j0 = threadIdx.x * kPer;
    i32x4u fs = {}, ps = {};
    if (j0 + kPer <= n) {
      fs = *reinterpret_cast<const i32x4u*>(a.fresh + s0 + j0);
      ps = *reinterpret_cast<const i32x4u*>(a.past + s0 + j0);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (j0 + i < n) fs[i] = a.fresh[s0 + j0 + i], ps[i] = a.past[s0 + j0 + i];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      at[i] = fresh[i] = min(max(fs[i], 0), most);
      past[i] = min(max(ps[i], 0), rows_most);
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
    __syncthreads();
    int top = 1;  // the greatest power of two below the number of sequences
    while (top * 2 < n) top *= 2;
    for (long t0 = ((long)(tokens / kTile - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x * (int)gridDim.x + (int)blockIdx.x) * kTile;
         t0 < tokens_end; t0 += (long)gridDim.x * kTile) {
      const int t = (int)t0 + (int)threadIdx.x;
      if (t < tokens || t >= tokens_end) continue;
      int seq = 0;  // the last sequence that begins at t or before
      for (int step = top; step > 0; step >>= 1)
        if (seq + step < n && begins[seq + step] <= t) seq += step;
      const int past = pasts[seq], pos = past + (t - begins[seq]);
      int slot = -1;
      if (pos < rows_most) {
        const int rank = (int)page.quot(pos), in = pos - rank * a.page_size, have = (int)page.quot(past + a.page_size - 1);
        const int j = news[seq] + rank - have;
        int32_t* entry = a.page_table + (s0 + seq) * (long)a.max_pages + rank;
        // the page's number: an old entry of the table, or the ring's
        const long k = ring.first + (long)j;
        const int32_t* from = rank < have ? entry : a.free_pages + (k >= a.n_free ? k - a.n_free : k);
        const int number = rank < have || j < ring.count ? *from : -1;
        if (rank >= have && in == 0) *entry = number;  // a new page's first token
        const long row = (long)number * a.page_size + in;
        slot = number < 0 || row > INT32_MAX ? -1 : (int)row;
      }
      a.pos[t] = pos;
      a.slots[t] = slot;
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
