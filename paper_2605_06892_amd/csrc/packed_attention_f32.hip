// fp32 attention of packed sequences with grouped heads, causal or not.
//
// Both contractions run on the matrix cores in fp32 (v_mfma_f32_16x16x4_f32),
// which bound it. One workgroup of 4 or 8 waves takes 16 rows (see packed.h)
// of one key/value head and its waves split the keys the tile sees (wave w
// takes the 32-key blocks w, w+NW, ...); their partial softmaxes are merged
// through LDS. Per 32-key block, in one wave:
//   S^T = K Q^T     K rows are the A operand (lane: key l%16), the queries the
//                   B operand. The contraction order is free, so a lane reads
//                   runs of 4 channels (16 bytes) and step 4j + t of slot l/16
//                   takes channel 16j + 4 (l/16) + t. Each lane then holds 8 scores
//                   of ONE row.
//   softmax         online; exp_neg is as exact as expf for x <= 0.
//   O^T += V^T P^T  step e takes the probabilities as they sit in the score
//                   registers (key row(e, slot)) and the matching rows of V;
//                   tile dt's row r is channel r*DT + dt, so a lane reads DT
//                   consecutive channels at once.
// Keys past the sequence read as zeros through the range check of a buffer
// resource that ends with the sequence.
#include "packed.h"

namespace hsa {
namespace {

constexpr int W = 16;      // rows per workgroup
constexpr int kKeys = 32;  // keys per block

__device__ __forceinline__ bool odd(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// NW: waves, each on its own key blocks
template <int DH, int NW>
__global__ __launch_bounds__(NW * kWave, DH == 64 ? 4 : 2) void packed_f32_kernel(PackedArgs a, PackedGrid grid) {
  constexpr int kThreads = NW * kWave;
  typedef typename Mfma<W>::acc Acc;
  constexpr int SL = kWave / W;        // contraction slots of one instruction
  constexpr int NE = W / SL;           // result registers per lane
  constexpr int KT = kKeys / W;        // key tiles of a block
  constexpr int DT = DH / W;           // channel tiles of O^T
  constexpr int J = DH / (4 * SL);     // 16-byte reads of a K or Q row per lane
  constexpr int CPR = DH / 4;          // 16-byte chunks per row
  constexpr int LD = kKeys * CPR / kWave;  // 16-byte loads per lane of a block's K rows
  constexpr int P = DH + 4;            // padded LDS row, floats
  typedef float vrow __attribute__((ext_vector_type(DT)));
  typedef vrow vrow_lds __attribute__((aligned(16)));
  static_assert(P * 4 % alignof(vrow_lds) == 0, "rows of the merge buffer are aligned for its stores");
  // per wave: its block's K rows, at the end its share of the output
  __shared__ __attribute__((aligned(16))) float buf[NW][kKeys * P];
  __shared__ float m_part[NW][W], l_part[NW][W];
  __shared__ int odd_part[NW];
  int h, idx;
  SeqTile t;
  packed_place(grid, h, idx);
  if (!find_tile<W>(a, idx, t)) return;

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lw = lane % W, slot = lane / W;
  const int n_rows = t.len_q * a.group, r0 = t.tile * W;
  const int seen = keys_seen(a, t, (int)a.by_group.quot(min(r0 + lw, n_rows - 1)));
  const int seen_lo = keys_seen(a, t, (int)a.by_group.quot(r0));
  const int seen_hi = keys_seen(a, t, (int)a.by_group.quot(min(r0 + W - 1, n_rows - 1)));
  const float* kg = static_cast<const float*>(a.k) + t.k0 * a.k_stride + (long)h * DH;
  const float* vg = static_cast<const float*>(a.v) + t.k0 * a.v_stride + (long)h * DH;

  // this lane's row (rows past the sequence repeat its last one and are not stored)
  f32x4 qf[J];
  {
    const int R = min(r0 + lw, n_rows - 1), i = (int)a.by_group.quot(R);
    const float* qr = static_cast<const float*>(a.q) + (t.q0 + i) * a.q_stride +
                      (long)(h * a.group + R - i * a.group) * DH + slot * 4;
#pragma unroll
    for (int j = 0; j < J; ++j) qf[j] = *reinterpret_cast<const f32x4u*>(qr + j * 4 * SL);
  }

  // Maxima are of the products q.k and the scale follows the subtraction: the
  // exponents (q.k - m) scale are at most 0 however large the products are.
  Acc acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (Acc){};
  float m_run = -INFINITY, l_run = 0.f;
  // Where a row does not see a key its weight is 0, but 0 times an infinite
  // value is NaN. In blocks that some row does not see whole, values that are not
  // finite are left out of the products, and the merge adds them to the rows that see them.
  bool cut_odd = false;

  // C channels of row n0 + r + step, c floats into it (r and c per lane, n0 and
  // step uniform), through a buffer resource from row n0 to the sequence's
  // end; where it may end inside the block, the step is part of the lane's
  // offset, the one that is range-checked
  auto read = [&](auto* dst, const float* base, int stride, int n0, int r, int step, int c) {
    constexpr int C = sizeof(*dst) / 4;
    const unsigned bytes = ((unsigned)(min(kKeys, t.len_k - n0) - 1) * stride + DH) * 4;
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base + (long)n0 * stride), 0, (int)bytes, 0x00020000);
    int vo = (r * stride + c) * 4, so = step * stride * 4;
    if (n0 + kKeys > t.len_k) {
      vo += so;
      so = 0;
    }
#pragma unroll
    for (int i = 0; i < C / 4; ++i) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rs, vo + i * 16, so, 0);
      __builtin_memcpy(reinterpret_cast<char*>(dst) + i * 16, &x, sizeof(x));
    }
  };

  // A block's K rows go to LDS through registers: loaded (whole rows, so that
  // every line is read once) during the previous block's softmax and PV, and
  // written just before its scores. Only this wave reads them: no barrier.
  float* kl = buf[wave];
  f32x4 kr[LD];
  auto load_k = [&](int n0) {
    if (n0 >= seen_hi) return;
#pragma unroll
    for (int i = 0; i < LD; ++i)
      read(&kr[i], kg, (int)a.k_stride, n0, lane / CPR, i * (kWave / CPR), lane % CPR * 4);
  };
  vrow vf[KT][NE];
  auto load_v = [&](int n0) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < NE; ++e)
        read(&vf[kt][e], vg, (int)a.v_stride, n0, Mfma<W>::row(0, slot), kt * W + Mfma<W>::row(e, 0), lw * DT);
  };
  load_k(wave * kKeys);
  for (int n0 = wave * kKeys; n0 < seen_hi; n0 += NW * kKeys) {
    const bool cut = n0 + kKeys > seen_lo;  // some row does not see every key of the block
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int f = i * kWave + lane;
      *reinterpret_cast<f32x4*>(&kl[(f / CPR) * P + (f % CPR) * 4]) = kr[i];
    }
    load_v(n0);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // the K rows are in LDS
    Acc s[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) s[kt] = (Acc){};
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const f32x4 kf = *reinterpret_cast<const f32x4*>(&kl[(kt * W + lw) * P + j * 4 * SL + slot * 4]);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[kt] = Mfma<W>::mul(kf[u], qf[j][u], s[kt]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // read before the next block's rows
    load_k(n0 + NW * kKeys);

    if (cut) {
      bool odd_v = false;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          if (n0 + kt * W + Mfma<W>::row(e, slot) >= seen) s[kt][e] = -INFINITY;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) odd_v |= odd(vf[kt][e][dt]);
        }
      if (__any(odd_v)) {  // see cut_odd
        cut_odd = true;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < NE; ++e)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[kt][e][dt] = odd(vf[kt][e][dt]) ? 0.f : vf[kt][e][dt];
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < NE; ++e) mx = fmaxf(mx, s[kt][e]);
#pragma unroll
    for (int x = W; x < kWave; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
    if (__any(mx > m_run)) {
      // raise the running maximum (wave-uniform branch, rare after the first blocks)
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : expf((m_run - m_new) * a.scale);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;  // no key or only -inf scores so far: weights 0
    float ls = 0.f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        s[kt][e] = exp_neg((s[kt][e] - m_use) * a.scale);
        ls += s[kt][e];
      }
    l_run += ls;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] = Mfma<W>::mul(vf[kt][e][dt], s[kt][e], acc[dt]);
  }

  // merge: the waves' softmaxes, each rescaled to the common maximum
  float l_tot = l_run;
#pragma unroll
  for (int x = W; x < kWave; x <<= 1) l_tot += __shfl_xor(l_tot, x);
  if (lane == 0) odd_part[wave] = cut_odd;
  if (slot == 0) {
    m_part[wave][lw] = m_run;
    l_part[wave][lw] = l_tot;
  }
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    vrow r;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) r[dt] = acc[dt][e];
    *reinterpret_cast<vrow_lds*>(&kl[lw * P + Mfma<W>::row(e, slot) * DT]) = r;
  }
  __syncthreads();
  bool any_odd = false;
#pragma unroll
  for (int w = 0; w < NW; ++w) any_odd |= odd_part[w] != 0;
  for (int f = threadIdx.x; f < W * CPR; f += kThreads) {
    const int r = f / CPR, c = (f - r * CPR) * 4;
    const int R = r0 + r;
    if (R >= n_rows) continue;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, m_part[w][r]);
    f32x4 sum = {};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = m_part[w][r];
      if (mw == -INFINITY && l_part[w][r] == 0.f) continue;  // no key, or no finite score
      const float wt = expf((mw - m) * a.scale);
      l = fmaf(wt, l_part[w][r], l);
      const f32x4 x = *reinterpret_cast<const f32x4*>(&buf[w][r * P + c]);
#pragma unroll
      for (int u = 0; u < 4; ++u) sum[u] = fmaf(wt, x[u], sum[u]);
    }
    sum *= l == 0.f ? 0.f : 1.f / l;
    const int i = (int)a.by_group.quot(R), hq = h * a.group + R - i * a.group;
    const long orow = (long)(t.q0 + i) * (a.kv_heads * a.group) + hq;
    if (any_odd && l != 0.f) {
      const int end = keys_seen(a, t, i);
      for (int n = max(seen_lo, 0) / kKeys * kKeys; n < end; ++n)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float x = vg[n * a.v_stride + c + u];
          if (odd(x)) sum[u] += x;
        }
    }
    *reinterpret_cast<f32x4u*>(static_cast<float*>(a.o) + orow * DH + c) = sum;
    if (a.lse && c == 0) a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, logf(l));
  }
}

template <int DH, int NW>
hipError_t launch_waves(const PackedArgs& a, hipStream_t s) {
  const PackedGrid g = packed_grid(a, W, DH * 4);
  if (g.groups < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_f32_kernel<DH, NW>), dim3((unsigned)g.groups), dim3(NW * kWave), 0, s, a, g);
  return hipGetLastError();
}

// 8 waves where few tiles leave a CU to each, 4 where the CUs share many: fitted to
// 444 launches like the bf16 form's tiles (see there), where the lesser estimate takes
// 1.3% more than the faster of the two on average. Measured with 64-wide heads, 4 and 8
// waves: 1 prompt of 1000 tokens, 1 head 19.1 and 17.1; 5 prompts of 33 to 700, 12 heads
// 34.7 and 38.9. (32 rows per workgroup, 8 waves: 27.7 and 47.7.)
constexpr PackedCost kCosts[2][2] = {{{W, 8, 3.6, 3.2, 0.329, 0.062}, {W, 4, 5.6, 1.25, 0.362, 0.115}},  // 64-wide heads
                                     {{W, 8, 0.0, 8.3, 0.697, 0.27}, {W, 4, 3.6, 4.6, 0.672, 0.804}}};  // 128-wide

template <int DH>
hipError_t launch_dh(const PackedArgs& a, hipStream_t s) {
  const PackedCost* c = packed_choice(a, kCosts[DH == 128]);
  if (!c) return hipErrorInvalidValue;
  return c->waves == 4 ? launch_waves<DH, 4>(a, s) : launch_waves<DH, 8>(a, s);
}

}  // namespace

hipError_t launch_packed_attention_f32(const PackedArgs& a, int head_dim, hipStream_t s) {
  return head_dim == 64 ? launch_dh<64>(a, s) : launch_dh<128>(a, s);
}

}  // namespace hsa
