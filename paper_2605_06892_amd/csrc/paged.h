// What the attention kernels over paged caches share: the dealing of the cached rows to workgroups, the parts
// that they leave, and the kernel that joins those.
#pragma once

#include "seq_common.h"

#include <algorithm>

namespace hsa {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 128;       // rows of a tile
constexpr int kRows = 16;        // query heads of an item
constexpr int kMostRuns = 1024;
constexpr int kJoinThreads = 256;

struct Plan {
  int wgs;        // runs of tiles, two parts to each
  int gts;        // items per (sequence, key/value head)
  FastDiv page;
  int runs;       // e2m1 rows: runs of each item (0: the tiles of all items in one order)
  int abreast;    // e2m1 rows: items that a workgroup takes at once
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int seq_len(const PagedArgs& a, int s) {
  const long most = a.n_pages > 0 ? (long)a.max_pages * a.page_size : 0;
  const int len = max(a.kv_lens[s], 0);
  return len > most ? (int)most : len;
}
// tiles of a sequence (one for an empty one: its output is written too)
__device__ __forceinline__ int tiles_of(int len) { return max((len + kTile - 1) / kTile, 1); }

// x / y for non-negative values, in 32 bits where they fit
__device__ __forceinline__ long div_pos(long x, long y) {
  return (x | y) >> 31 ? x / y : (long)((unsigned)x / (unsigned)y);
}

// The tiles of all items in order: sequence by sequence, in it head by head. A
// wave's view: 64 sequences at a time, the whole batch at once where it has no more.
struct Walk {
  int s0;           // first sequence in view
  int len;          // of sequence s0 + lane
  long before;      // tiles before s0
  long from, upto;  // tiles before and up to the end of this lane's sequence

  __device__ __forceinline__ void view(const PagedArgs& a, int per, int first, long tiles_before) {
    const int lane = threadIdx.x & (kWave - 1);
    s0 = first;
    before = tiles_before;
    len = s0 + lane < a.n_seqs ? seq_len(a, s0 + lane) : 0;
    const long n = s0 + lane < a.n_seqs ? (long)tiles_of(len) * per : 0;
    upto = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const long y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    upto += before;
    from = upto - n;
  }
  __device__ __forceinline__ long end() const { return __shfl(upto, kWave - 1); }
  // Lane whose sequence holds tile `at`, moving the view on to it; -1 past the last sequence.
  __device__ __forceinline__ int find(const PagedArgs& a, int per, long at) {
    for (;;) {
      const unsigned long hit = __ballot(from <= at && at < upto);
      if (hit) return __builtin_ctzl(hit);
      if (s0 + kWave >= a.n_seqs) return -1;
      view(a, per, s0 + kWave, end());
    }
  }
};

// tiles of all items
__device__ __forceinline__ long all_tiles(const PagedArgs& a, int per, const Walk& first) {
  if (a.n_seqs <= kWave) return first.end();
  long sum = 0;
  for (int s = threadIdx.x & (kWave - 1); s < a.n_seqs; s += kWave) sum += tiles_of(seq_len(a, s));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  return sum * per;
}
// tiles of a run
__device__ __forceinline__ long run_tiles(long total, int wgs) { return div_pos(total + wgs - 1, wgs); }

template <int DH>
struct Part {  // a part of an item in the workspace
  float o[kRows * DH];
  float ml[kRows * 2];
};
// The item that a run begins and does not end: its parts are this run's in
// `slot` and the next `more` runs' first (0: there is no such item). In the workspace
// behind the parts, two to a run.
struct Note {
  int s, item, slot, more;
};
template <int DH>
__device__ __forceinline__ Note* notes(const PagedArgs& a, const Plan& plan) {
  return reinterpret_cast<Note*>(static_cast<Part<DH>*>(a.ws) + 2 * (long)plan.wgs);
}

// exp((x - y) * scale) for x <= y, as exact as the form needs
template <bool F32>
__device__ __forceinline__ float rescale(float x, float y, float scale) {
  return F32 ? expf((x - y) * scale) : __builtin_amdgcn_exp2f((x - y) * (scale * kLog2e));
}

// 4 channels (from c) of query head `orow` of all, and with c == 0 its lse, from
// the softmax's maximum, sum and weighted values
template <bool F32, int DH>
__device__ __forceinline__ void write_out(const PagedArgs& a, long orow, int c, float m, float l, f32x4 sum) {
  sum *= l == 0.f ? 0.f : 1.f / l;
  if constexpr (F32) *reinterpret_cast<f32x4u*>(static_cast<float*>(a.o) + orow * DH + c) = sum;
  else *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + orow * DH + c) = to_bf16x4(sum);
  if (a.lse && c == 0) a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, logf(l));
}

// The output of query head r of the item that run w0 begins and does not end, by a workgroup: its threads take 4 channels
// each of every few parts, then join those.
template <bool F32, int DH>
__device__ __forceinline__ void join_parts(const PagedArgs& a, const Plan& plan, const Note& note, int w0, int r) {
  constexpr int C = DH / 4, G = kJoinThreads / C;  // threads per part, parts at a time
  __shared__ __attribute__((aligned(16))) f32x4 sums[G][C];
  __shared__ float ms[G], ls[G];
  const int h = note.item / plan.gts, g = (note.item - h * plan.gts) * kRows + r;
  if (g >= a.group) return;
  const Part<DH>* parts = static_cast<const Part<DH>*>(a.ws);
  const int lane_p = threadIdx.x / C, c = (threadIdx.x - lane_p * C) * 4;
  float m = -INFINITY, l = 0.f;
  f32x4 sum = {};
  constexpr int U = 4;  // parts loaded at once by each
  for (int i0 = lane_p; i0 <= note.more; i0 += U * G) {
    f32x2 ml[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * G, note.more);
      const Part<DH>* p = parts + 2 * (long)(w0 + i) + (i ? 0 : note.slot);
      ml[u] = *reinterpret_cast<const f32x2*>(&p->ml[2 * r]);
      x[u] = *reinterpret_cast<const f32x4*>(&p->o[r * DH + c]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * G > note.more || (ml[u][0] == -INFINITY && ml[u][1] == 0.f)) continue;  // no key, or no finite score
      const float m_new = fmaxf(m, ml[u][0]);
      const float was = m == -INFINITY ? 0.f : rescale<F32>(m, m_new, a.scale), wt = rescale<F32>(ml[u][0], m_new, a.scale);
      m = m_new;
      l = fmaf(wt, ml[u][1], l * was);
      sum = sum * was + wt * x[u];
    }
  }
  sums[lane_p][c / 4] = sum;
  if (c == 0) {
    ms[lane_p] = m;
    ls[lane_p] = l;
  }
  __syncthreads();
  if (lane_p > 0) return;
  float m_all = -INFINITY;
#pragma unroll
  for (int i = 0; i < G; ++i) m_all = fmaxf(m_all, ms[i]);
  l = 0.f;
  sum = (f32x4){};
#pragma unroll
  for (int i = 0; i < G; ++i) {
    if (ms[i] == -INFINITY && ls[i] == 0.f) continue;
    const float wt = rescale<F32>(ms[i], m_all, a.scale);
    l = fmaf(wt, ls[i], l);
    sum += wt * sums[i][c / 4];
  }
  write_out<F32, DH>(a, (long)note.s * (a.kv_heads * a.group) + h * a.group + g, c, m_all, l, sum);
}

// One query head (blockIdx.y) of an item that a run begins and does not end. FEW: blockIdx.x counts those items, and the run is
// found by looking through all notes; else it is the run, and its workgroup may find nothing to do. Sending out workgroups for
// nothing takes 1 to 3 us for 512 to 1024 runs, so they are counted where there are 32 runs to an item or more. Counted, one for
// each run, and eight runs to a workgroup, which joins what they begin in turn, us:
//                                                                      counted   each   eight
//     4 sequences of 30011 to 131072 e2m1 rows, 40/8 heads               72.7    74.5   72.5
//     2 of 131072 bf16 rows, 40/8                                         189     191    189
//     16 of 65536 e4m3 rows, 16/1                                        49.4    56.5   50.0
//     16 of 200 bf16 rows in a table of 131072, 16/1                     11.4    12.0   15.2
//     2 of 200 bf16 rows in a table of 131072, 40/8                      10.5    11.0   13.9
template <bool F32, int DH, bool FEW>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedArgs a, Plan plan) {
  if constexpr (!FEW) {
    const Note note = notes<DH>(a, plan)[blockIdx.x];
    if (note.more != 0) join_parts<F32, DH>(a, plan, note, blockIdx.x, blockIdx.y);
  } else {
    constexpr int W = kJoinThreads / kWave, N = kMostRuns / kJoinThreads;  // a wave looks through N times 64 notes
    __shared__ int begins[W], at;  // items that the runs of each wave begin; the run sought
    __shared__ Note found;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, first = wave * (N * kWave) + lane;
    Note own[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      own[i] = Note{0, 0, 0, 0};
      if (first + i * kWave < plan.wgs) own[i] = notes<DH>(a, plan)[first + i * kWave];
    }
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __builtin_popcountl(__ballot(own[i].more != 0));
    if (lane == 0) begins[wave] = n;
    if (threadIdx.x == 0) at = -1;
    __syncthreads();
    int rank = -(int)blockIdx.x;  // of the next item, from the one sought
#pragma unroll
    for (int w = 0; w < W; ++w) rank += w < wave ? begins[w] : 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned long some = __ballot(own[i].more != 0);
      const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(some >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)some, 0));
      if (own[i].more != 0 && rank + before == 0) {
        found = own[i];
        at = first + i * kWave;
      }
      rank += __builtin_popcountl(some);
    }
    __syncthreads();
    const int run = uniform(at);
    const Note note{uniform(found.s), uniform(found.item), uniform(found.slot), uniform(found.more)};
    if (run >= 0) join_parts<F32, DH>(a, plan, note, run, blockIdx.y);
  }
}
template <bool F32, int DH>
hipError_t launch_join(const PagedArgs& a, const Plan& plan, hipStream_t s) {
  const unsigned rows = std::min(a.group, kRows);
  const long items = (long)a.n_seqs * a.kv_heads * plan.gts;
  if (plan.wgs >= 32 * items)
    hipLaunchKernelGGL((paged_join_kernel<F32, DH, true>), dim3((unsigned)items, rows), dim3(kJoinThreads), 0, s, a, plan);
  else
    hipLaunchKernelGGL((paged_join_kernel<F32, DH, false>), dim3(plan.wgs, rows), dim3(kJoinThreads), 0, s, a, plan);
  return hipGetLastError();
}

inline int gts_of(int group) { return (group + kRows - 1) / kRows; }

// Rows up to which an item is one workgroup's. Dealing out tiles costs the walk and the join
// (4 to 5 us), a whole item the time of its rows in one workgroup, and the fewer items, the
// fewer CUs share that. Whole and dealt, us, bf16, 128 channels, batches of half to full length:
//     8 items    700 rows 11.1  9.8    1000 14.6  9.7    1500 19.9 10.1
//    64          700      11.8 11.8    1000 15.7 12.6    1500 21.3 16.2
//   128         1000      16.7 19.1    1250 19.4 19.3    2000 28.0 25.4
//   256         1000      20.6 26.0    2000 35.7 38.3    4000 73.5 75.4
// (64 channels and e4m3 cross within a third of these. e2m1 rows cross further out: 64 items of 700 rows 7.9 13.2, 128 of 1000 9.2
// 15.0, 256 of 2000 15.4 25.0, 512 of 2000 27.5 32.7. They are dealt from the same lengths on as the others.)
constexpr long kLeastWhole = 768;
inline long whole_len(long items) {
  const int cus = compute_units();
  return items * 4 <= cus ? kLeastWhole : items * 2 <= cus ? 1024 : 2048;
}
inline bool splits(int n_seqs, int kv_heads, int group, long max_len) {
  return max_len > whole_len((long)n_seqs * kv_heads * gts_of(group));
}

// Workgroups the tiles are dealt to: as many as run at once, no more than tiles
// if every sequence is as long as it may be.
inline int workgroups(int n_seqs, int kv_heads, int group, long max_len) {
  const long tiles = (long)n_seqs * kv_heads * gts_of(group) * ((max_len + kTile - 1) / kTile);
  return (int)std::min(std::min((long)kMostRuns, 2L * compute_units()), tiles);
}

}  // namespace

// Over e2m1 rows (paged_attention_e2m1.hip).
hipError_t launch_paged_attention_e2m1(const PagedArgs& a, bool bf16, int head_dim, hipStream_t s);

}  // namespace hsa
