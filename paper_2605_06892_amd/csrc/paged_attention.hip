// Attention of one query per sequence over a paged cache of bf16, fp32 or e4m3
// rows, with grouped heads. It reads every cached row of a key/value head once for
// all the query heads of its group, and that reading bounds it.
//
// Work split. An item is (sequence, key/value head, 16 query heads of its group); its rows
// come in tiles of 128. All tiles of all items, in order, are dealt to the
// workgroups in equal runs, so that a batch of very different lengths loads the CUs
// evenly and one long sequence is spread over all of them. A run that holds a whole item
// writes its output; the first and the last item of a run may be parts, which
// go to the workspace (unnormalized output, maximum and sum of the softmax) and are
// joined by a second kernel. Where each item begins follows from the lengths alone, and both
// kernels work it out for themselves: no atomics, no state between calls.
//
// In a workgroup, wave w of 4 takes the blocks w, w + 4, ... of its rows, 32 keys
// of bf16 or e4m3 rows (16 with fp32 queries), one block loaded ahead, with its own running
// softmax; the four are merged in LDS at the end of an item. The 16 query heads
// are one column tile of the matrix instructions, in S^T = K Q^T and, with the
// probabilities as they sit in the score registers, in O^T += V^T P^T.
//   bf16   16x16x32: K rows in the A operand's layout straight from global
//          memory, V rows through LDS for the transpose read. e4m3 rows become bf16 first,
//          without a rounding (4 significant bits and a power of two).
//   fp32   16x16x4: K and V rows both in their operand's layout.
// Probabilities are rounded to bf16 in the bf16 form; the sums take them before that.
#include "seq_common.h"

namespace hsa {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kTile = 128;    // rows of a tile
constexpr int kRows = 16;     // query heads of an item
constexpr int kMaxGroups = 1024;

struct Plan {
  int wgs;        // workgroups that the tiles are dealt to
  int gts;        // items per (sequence, key/value head)
  FastDiv page;
};

// tiles of a sequence (one for an empty one: its output is written too)
__device__ __forceinline__ int seq_tiles(const PagedArgs& a, int s, int& len) {
  const long most = a.n_pages > 0 ? (long)a.max_pages * a.page_size : 0;
  len = max(a.kv_lens[s], 0);
  if (len > most) len = (int)most;
  return max((len + kTile - 1) / kTile, 1);
}

// sum of seq_tiles over the sequences, by the whole workgroup
__device__ __forceinline__ long wg_total(const PagedArgs& a, long* lds) {
  long sum = 0;
  for (int s = threadIdx.x; s < a.n_seqs; s += kThreads) {
    int len;
    sum += seq_tiles(a, s, len);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += lds[w];
  return sum;
}
// The sequence that holds tile `at` of all items (a sequence has `per` items), searched
// from sequence s0 on, with `before` tiles before that; by one wave.
struct Found {
  long before;
  int seq;
};
__device__ __forceinline__ Found find_seq(const PagedArgs& a, int per, int s0, long before, long at) {
  const int lane = threadIdx.x & 63;
  for (; s0 < a.n_seqs; s0 += kWave) {
    int len;
    const long n = s0 + lane < a.n_seqs ? (long)seq_tiles(a, s0 + lane, len) * per : 0;
    long upto = n;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const long y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned long hit = __ballot(at < before + upto);
    if (hit) {
      const int l = __builtin_ctzl(hit);
      return {before + __shfl(upto - n, l), s0 + l};
    }
    before += __shfl(upto, kWave - 1);
  }
  return {before, a.n_seqs};
}

// first tile of workgroup w's run, and the run that holds a tile
__device__ __forceinline__ long run_begin(long total, int wgs, int w) { return total * w / wgs; }
__device__ __forceinline__ int run_of(long total, int wgs, long tile) { return (int)(((tile + 1) * wgs - 1) / total); }

template <int DH>
struct Part {  // a part of an item in the workspace
  float o[kRows * DH];
  float ml[kRows * 2];
};

template <bool F32, bool E4M3, int DH, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void paged_kernel(PagedArgs a, Plan plan) {
  constexpr int BK = F32 ? 16 : 32;        // keys per block
  constexpr int KT = BK / 16;              // key tiles of a block
  constexpr int DT = DH / 16;              // channel tiles of O^T
  constexpr int P = DH + 4;                // padded row of the merge buffer, floats
  constexpr int ES = E4M3 ? 1 : (F32 ? 4 : 2);
  constexpr int CB = 16;                   // bytes of a load
  constexpr int CE = CB / ES;              // values of a load
  constexpr int KL = DH / CE / 4;          // K loads per lane and key tile (its 4 slots share a row)
  // V: bf16 form, whole rows over the wave; fp32 form, DT consecutive channels of the 4 keys of a slot
  constexpr int VR = F32 ? 4 : BK * DH / CE / 64;
  constexpr int VB = F32 ? DT * ES : CB;   // bytes of one V read
  constexpr int CPR = DH / CE;             // loads per row
  struct VLoad { unsigned char b[VB]; };
  __shared__ __attribute__((aligned(16))) float buf[kWaves][kRows * P];  // V rows, then the merge
  __shared__ float m_part[kWaves][kRows], l_part[kWaves][kRows];
  __shared__ long sums[kWaves];
  static_assert(F32 || kRows * P * 4 >= BK * DH * 2, "a block's V rows fit");

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, grp = lane >> 4;
  const int per = a.kv_heads * plan.gts;
  const long total = wg_total(a, sums) * per;
  const int w = blockIdx.x;
  const long begin = run_begin(total, plan.wgs, w), end = run_begin(total, plan.wgs, w + 1);
  const int d_kv = a.kv_heads * DH;
  const float sl2e = a.scale * kLog2e;
  bf16* vl = reinterpret_cast<bf16*>(buf[wave]);
  auto swz = [](int r) { return DH == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1; };

  Found at{0, 0};
  for (long pos = begin; pos < end;) {
    at = find_seq(a, per, at.seq, at.before, pos);
    const int s = __builtin_amdgcn_readfirstlane(at.seq);
    if (s >= a.n_seqs) break;  // lengths that changed under the call
    int len;
    const int tiles = seq_tiles(a, s, len);
    const int item = (int)((pos - at.before) / tiles);
    const int t0 = (int)(pos - at.before - (long)item * tiles);
    const int n_t = (int)min((long)(tiles - t0), end - pos);
    const int h = item / plan.gts, g0 = (item - h * plan.gts) * kRows;
    const int key0 = t0 * kTile, key1 = min(len, key0 + n_t * kTile);
    const int32_t* pages = a.page_table + (long)s * a.max_pages;

    // this lane's query head (heads past the group repeat its last one and are not stored)
    const int hq = h * a.group + min(g0 + l16, a.group - 1);
    const long q_at = s * a.q_stride + (long)hq * DH;
    // the channels of slot grp at K load i, CE at a time: i*4*CE + grp*CE ..
    bf16x8 qb[F32 ? 1 : DH / 32];
    float qs[F32 ? DH / 4 : 1];
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < KL; ++i)
#pragma unroll
        for (int j = 0; j < CE; j += 4) {
          const f32x4u x = *reinterpret_cast<const f32x4u*>(static_cast<const float*>(a.q) + q_at + (i * 4 + grp) * CE + j);
#pragma unroll
          for (int u = 0; u < 4; ++u) qs[i * CE + j + u] = x[u];
        }
    } else {
#pragma unroll
      for (int i = 0; i < KL; ++i)
#pragma unroll
        for (int j = 0; j < CE / 8; ++j)
          qb[i * (CE / 8) + j] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.q) + q_at + (i * 4 + grp) * CE + j * 8);
    }

    f32x4 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){};
    float m_run = -INFINITY, l_run = 0.f;

    // one block ahead: its rows (as held), exponents, and which of its keys exist
    u32x4 kr[KT][KL];
    VLoad vr[VR];
    int ke[KT], ve[VR];
    unsigned mask = 0;
    // row of the cache that holds this lane's key of the block at n0 (lane % BK), -1 for none
    auto resolve = [&](int n0) -> int {
      const int t = n0 + (ALIGNED ? 0 : lane % BK);
      if (t >= key1) return -1;
      const int p = (int)plan.page.quot(t);
      const int page = pages[p];
      return page >= 0 && page < a.n_pages ? page * a.page_size + (t - p * a.page_size) : -1;
    };
    auto v_key = [&](int i) { return F32 ? grp * 4 + i : (i * 64 + lane) / CPR; };
    int row = resolve(key0 + wave * BK);
    auto load = [&](int n0) {
      if (n0 >= key1) return;
      int first = row;
      if constexpr (ALIGNED) {  // a block lies in one page: rows first ..
        first = __builtin_amdgcn_readfirstlane(row);
        const int n = key1 - n0;
        mask = first < 0 ? 0u : (n >= BK ? (BK == 32 ? ~0u : 0xffffu) : (1u << n) - 1);
        first = max(first, 0);
      } else {
        mask = (unsigned)__ballot(row >= 0) & (BK == 32 ? ~0u : 0xffffu);
        first = max(row, 0);
      }
      auto key_row = [&](int k) -> long { return ALIGNED ? first + k : __shfl(first, k); };
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const long r = key_row(kt * 16 + l16);
        const char* src = static_cast<const char*>(a.k) + (r * d_kv + h * DH + grp * CE) * ES;
#pragma unroll
        for (int i = 0; i < KL; ++i) __builtin_memcpy(&kr[kt][i], src + i * 4 * CB, CB);
        if constexpr (E4M3) ke[kt] = a.k_exp[r * a.kv_heads + h];
      }
#pragma unroll
      for (int i = 0; i < VR; ++i) {
        const long r = key_row(v_key(i));
        const int c = F32 ? l16 * DT : ((i * 64 + lane) % CPR) * CE;
        __builtin_memcpy(&vr[i], static_cast<const char*>(a.v) + (r * d_kv + h * DH + c) * ES, VB);
        if constexpr (E4M3) ve[i] = a.v_exp[r * a.kv_heads + h];
      }
      row = resolve(n0 + kWaves * BK);
    };
    load(key0 + wave * BK);

    for (int n0 = key0 + wave * BK; n0 < key1; n0 += kWaves * BK) {
      const unsigned keys = mask;
      const bool cut = keys != (BK == 32 ? ~0u : 0xffffu);
      f32x4 sc[KT] = {};
      float vf[F32 ? 4 : 1][DT];
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < KL; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x[CE / 4];
            if constexpr (E4M3) {
              const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[0][i][j], false);
              const f32x2 up = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[0][i][j], true);
              x[0] = lo[0], x[1] = lo[1], x[2] = up[0], x[3] = up[1];
            } else {
              x[0] = __uint_as_float(kr[0][i][j]);
            }
#pragma unroll
            for (int u = 0; u < CE / 4; ++u)
              sc[0] = Mfma<16>::mul(x[u], qs[i * CE + j * (CE / 4) + u], sc[0]);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (E4M3) {
            const float sv = pow2(ve[i]);
#pragma unroll
            for (int j = 0; j < DT / 4; ++j) {
              int c;
              __builtin_memcpy(&c, &vr[i].b[j * 4], 4);
              const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), up = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
              vf[i][j * 4] = lo[0] * sv, vf[i][j * 4 + 1] = lo[1] * sv;
              vf[i][j * 4 + 2] = up[0] * sv, vf[i][j * 4 + 3] = up[1] * sv;
            }
          } else {
            __builtin_memcpy(vf[i], &vr[i], VB);
          }
          if (cut && !(keys >> v_key(i) & 1))
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[i][dt] = 0.f;
        }
        if constexpr (E4M3) {  // the keys' exponents, from the lanes that loaded them
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[0][e] *= pow2(__shfl(ke[0], grp * 4 + e));
        }
      } else {
#pragma unroll
        for (int i = 0; i < VR; ++i) {
          const int f = i * 64 + lane, r = f / CPR;
          u32x4 x;
          __builtin_memcpy(&x, &vr[i], CB);
          if (cut && !(keys >> r & 1)) x = (u32x4){};
          if constexpr (E4M3) {
            const float sv = pow2(ve[i]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              bf16x8 y;
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * j + u], sv, false);
                const bf16x2 up = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * j + u], sv, true);
                y[4 * u] = lo[0], y[4 * u + 1] = lo[1], y[4 * u + 2] = up[0], y[4 * u + 3] = up[1];
              }
              *reinterpret_cast<bf16x8*>(vl + r * DH + ((((f % CPR) * 2 + j) ^ swz(r)) * 8)) = y;
            }
          } else {
            *reinterpret_cast<u32x4*>(vl + r * DH + ((f % CPR) ^ swz(r)) * 8) = x;
          }
        }
#pragma unroll
        for (int i = 0; i < KL; ++i)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            if constexpr (E4M3) {
              const float sk = pow2(ke[kt]);
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                bf16x8 y;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kr[kt][i][2 * j + u], sk, false);
                  const bf16x2 up = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kr[kt][i][2 * j + u], sk, true);
                  y[4 * u] = lo[0], y[4 * u + 1] = lo[1], y[4 * u + 2] = up[0], y[4 * u + 3] = up[1];
                }
                sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, qb[i * 2 + j], sc[kt], 0, 0, 0);
              }
            } else {
              sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[kt][i]), qb[i], sc[kt], 0, 0, 0);
            }
          }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // the V rows are in LDS
      }
      load(n0 + kWaves * BK);

      if (cut) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(keys >> (kt * 16 + grp * 4 + e) & 1)) sc[kt][e] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, sc[kt][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__any(mx > m_run)) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_run == -INFINITY ? 0.f : (F32 ? expf((m_run - m_new) * a.scale) : __builtin_amdgcn_exp2f((m_run - m_new) * sl2e));
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
        m_run = m_new;
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;  // no key or only -inf scores so far: weights 0
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[kt][e] = F32 ? exp_neg((sc[kt][e] - m_use) * a.scale) : __builtin_amdgcn_exp2f((sc[kt][e] - m_use) * sl2e);
          l_run += sc[kt][e];
        }
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt] = Mfma<16>::mul(vf[e][dt], sc[0][e], acc[dt]);
      } else {
        const bf16x8 pf = __builtin_shufflevector(to_bf16x4(sc[0]), to_bf16x4(sc[KT - 1]), 0, 1, 2, 3, 4, 5, 6, 7);
        const int r = grp * 4 + (l16 >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int col = dt * 16 + 4 * (lane & 3);
          const bf16* src = vl + r * DH + (((col >> 3) ^ swz(r)) * 8) + (col & 7);
          const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src));
          const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src + 16 * DH));
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pf,
                                                            acc[dt], 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // read before the next block's rows
      }
    }

    // merge of the waves. acc[dt][e] is channel dt*16 + grp*4 + e of row l16,
    // in the fp32 form (grp*4 + e)*DT + dt
    float l_tot = l_run + __shfl_xor(l_run, 16);
    l_tot += __shfl_xor(l_tot, 32);
    if (grp == 0) {
      m_part[wave][l16] = m_run;
      l_part[wave][l16] = l_tot;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) buf[wave][l16 * P + (grp * 4 + e) * DT + dt] = acc[dt][e];
      } else {
        *reinterpret_cast<f32x4*>(&buf[wave][l16 * P + dt * 16 + grp * 4]) = acc[dt];
      }
    }
    __syncthreads();
    const bool whole = n_t == tiles;
    Part<DH>* part = static_cast<Part<DH>*>(a.ws) + 2 * (long)w + (pos == begin ? 0 : 1);
    const int n_heads = min(kRows, a.group - g0);
    for (int f = threadIdx.x; f < n_heads * (DH / 4); f += kThreads) {
      const int r = f / (DH / 4), c = (f - r * (DH / 4)) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) m = fmaxf(m, m_part[x][r]);
      f32x4 sum = {};
      float l = 0.f;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float mw = m_part[x][r];
        if (mw == -INFINITY && l_part[x][r] == 0.f) continue;  // no key, or no finite score
        const float wt = F32 ? expf((mw - m) * a.scale) : __builtin_amdgcn_exp2f((mw - m) * sl2e);
        l = fmaf(wt, l_part[x][r], l);
        sum += wt * *reinterpret_cast<const f32x4*>(&buf[x][r * P + c]);
      }
      if (whole) {
        sum *= l == 0.f ? 0.f : 1.f / l;
        const long orow = (long)s * (a.kv_heads * a.group) + h * a.group + g0 + r;
        if constexpr (F32) *reinterpret_cast<f32x4u*>(static_cast<float*>(a.o) + orow * DH + c) = sum;
        else *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + orow * DH + c) = to_bf16x4(sum);
        if (a.lse && c == 0) a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, logf(l));
      } else {
        *reinterpret_cast<f32x4*>(&part->o[r * DH + c]) = sum;
        if (c == 0) *reinterpret_cast<f32x2*>(&part->ml[2 * r]) = (f32x2){m, l};
      }
    }
    __syncthreads();  // the merge has read what the next item writes
    pos += n_t;
  }
}

// Items that more than one run holds: their parts, rescaled to the common
// maximum. One workgroup per item.
template <bool F32, int DH>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(PagedArgs a, Plan plan) {
  const int per = a.kv_heads * plan.gts;
  const int s = blockIdx.x / per, item = blockIdx.x - s * per;
  long before = 0, all = 0;
  for (int i = threadIdx.x & 63; i < a.n_seqs; i += kWave) {
    int len;
    const int n = seq_tiles(a, i, len);
    all += n;
    if (i < s) before += n;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    all += __shfl_xor(all, o);
    before += __shfl_xor(before, o);
  }
  int len;
  const int tiles = seq_tiles(a, s, len);
  const long total = all * per, first = before * per + (long)item * tiles;
  const int w0 = run_of(total, plan.wgs, first), w1 = run_of(total, plan.wgs, first + tiles - 1);
  if (w0 == w1) return;
  const Part<DH>* parts = static_cast<const Part<DH>*>(a.ws);
  auto part = [&](int w) { return parts + 2 * (long)w + (w > w0 || run_begin(total, plan.wgs, w) == first ? 0 : 1); };
  const int h = item / plan.gts, g0 = (item - h * plan.gts) * kRows;
  const int n_heads = min(kRows, a.group - g0);
  const float sl2e = a.scale * kLog2e;
  for (int f = threadIdx.x; f < n_heads * (DH / 4); f += kThreads) {
    const int r = f / (DH / 4), c = (f - r * (DH / 4)) * 4;
    float m = -INFINITY, l = 0.f;
    f32x4 sum = {};
    for (int w = w0; w <= w1; ++w) {
      if (w > w0 && run_begin(total, plan.wgs, w) == run_begin(total, plan.wgs, w + 1)) continue;  // an empty run
      const Part<DH>* p = part(w);
      const f32x2 ml = *reinterpret_cast<const f32x2*>(&p->ml[2 * r]);
      if (ml[0] == -INFINITY && ml[1] == 0.f) continue;
      const float m_new = fmaxf(m, ml[0]);
      const float was = m == -INFINITY ? 0.f : (F32 ? expf((m - m_new) * a.scale) : __builtin_amdgcn_exp2f((m - m_new) * sl2e));
      const float wt = F32 ? expf((ml[0] - m_new) * a.scale) : __builtin_amdgcn_exp2f((ml[0] - m_new) * sl2e);
      m = m_new;
      l = fmaf(wt, ml[1], l * was);
      sum = sum * was + wt * *reinterpret_cast<const f32x4*>(&p->o[r * DH + c]);
    }
    sum *= l == 0.f ? 0.f : 1.f / l;
    const long orow = (long)s * (a.kv_heads * a.group) + h * a.group + g0 + r;
    if constexpr (F32) *reinterpret_cast<f32x4u*>(static_cast<float*>(a.o) + orow * DH + c) = sum;
    else *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + orow * DH + c) = to_bf16x4(sum);
    if (a.lse && c == 0) a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, logf(l));
  }
}

int gts_of(int group) { return (group + kRows - 1) / kRows; }
long tiles_most(long max_len) { return max_len > kTile ? (max_len + kTile - 1) / kTile : 1; }

// Workgroups the tiles are dealt to: as many as run at once, no more than tiles
// if every sequence is as long as it may be.
int workgroups(int n_seqs, int kv_heads, int group, long max_len) {
  const long items = (long)n_seqs * kv_heads * gts_of(group);
  const long most = std::min((long)kMaxGroups, 2L * compute_units());
  return (int)std::min(most, items * tiles_most(max_len));
}

template <bool F32, bool E4M3, int DH>
hipError_t launch(const PagedArgs& a, hipStream_t s) {
  const long max_len = (long)a.max_pages * a.page_size;
  Plan plan{workgroups(a.n_seqs, a.kv_heads, a.group, max_len), gts_of(a.group), FastDiv((uint32_t)a.page_size)};
  if (a.page_size % 32 == 0)
    hipLaunchKernelGGL((paged_kernel<F32, E4M3, DH, true>), dim3(plan.wgs), dim3(kThreads), 0, s, a, plan);
  else
    hipLaunchKernelGGL((paged_kernel<F32, E4M3, DH, false>), dim3(plan.wgs), dim3(kThreads), 0, s, a, plan);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || tiles_most(max_len) == 1) return e;
  hipLaunchKernelGGL((paged_join_kernel<F32, DH>), dim3((unsigned)(a.n_seqs * a.kv_heads * plan.gts)), dim3(kThreads), 0, s, a, plan);
  return hipGetLastError();
}

template <bool F32, int DH>
hipError_t launch_held(const PagedArgs& a, bool e4m3, hipStream_t s) {
  return e4m3 ? launch<F32, true, DH>(a, s) : launch<F32, false, DH>(a, s);
}

}  // namespace

size_t paged_attention_bytes(int n_seqs, int kv_heads, int group, int head_dim, long max_len) {
  if (n_seqs <= 0 || tiles_most(max_len) == 1) return 0;
  return (size_t)workgroups(n_seqs, kv_heads, group, max_len) * 2 * kRows * (head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedArgs& a, bool bf16, bool e4m3, int head_dim, hipStream_t s) {
  if (a.n_seqs <= 0) return hipSuccess;
  if (bf16) return head_dim == 64 ? launch_held<false, 64>(a, e4m3, s) : launch_held<false, 128>(a, e4m3, s);
  return head_dim == 64 ? launch_held<true, 64>(a, e4m3, s) : launch_held<true, 128>(a, e4m3, s);
}

}  // namespace hsa
