// bf16 attention of packed sequences with grouped heads, causal or not.
//
//   o_i = sum_j softmax_j(scale <q_i, k_j>) v_j over the keys that query i sees
//
// Small tiles (this file): 16 or 32 rows (see packed.h) of one key/value head per
// workgroup, whose 4 or 8 waves split the keys (wave w takes the 32-key blocks w,
// w+NW, ...) and merge their softmaxes in LDS; no wave waits for another before
// that. Per block of a wave: S^T = K Q^T by v_mfma_f32_16x16x32_bf16 (32x32x16 for 32
// rows), K rows straight from global memory in the A operand's layout; each lane holds
// scores of ONE row, which are the B operand of O^T += V^T P^T as they sit. V
// rows go through the wave's LDS region for the transpose read. Both are loaded one
// block ahead.
//
// Scores are exact products of the bf16 inputs, and the scale follows the
// subtraction of the running maximum in fp32. Rounded to bf16 are the probabilities
// (the sum takes them before that) and the output.
#include "packed.h"
#include "packed_tile.h"

namespace hsa {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kKeys = 32;  // keys per block

// The W x W bf16 matrix instruction: 64/W contraction slots (lane / W) of 8
// values, the result's column lane % W, its rows row(e, lane / W).
template <int W>
struct MfmaB;
template <>
struct MfmaB<16> {
  typedef f32x4 acc;
  static __device__ __forceinline__ acc mul(bf16x8 a, bf16x8 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct MfmaB<32> {
  typedef f32x16 acc;
  static __device__ __forceinline__ acc mul(bf16x8 a, bf16x8 b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// W: rows per workgroup, NW: its waves
template <int DH, int W, int NW>
__global__ __launch_bounds__(NW * 64) void packed_small_kernel(PackedArgs a, PackedGrid grid) {
  typedef typename MfmaB<W>::acc Acc;
  constexpr int SL = 64 / W;               // contraction slots
  constexpr int NE = W / SL;               // result registers per lane
  constexpr int KT = kKeys / W;            // key tiles of a block
  constexpr int KK = DH / (8 * SL);        // k-steps of S^T
  constexpr int DT = DH / W;               // head-dim tiles of O^T
  constexpr int KS = kKeys / (8 * SL);     // k-steps of O^T
  constexpr int CPR = DH / 8;              // 16-byte chunks per row
  constexpr int LV = kKeys * CPR / 64;     // V loads per lane and block
  constexpr int P = DH + 4;                // padded row of the merge buffer, floats
  __shared__ __attribute__((aligned(16))) float buf[NW][W * P];  // V rows, then the merge
  __shared__ float m_part[NW][W], l_part[NW][W];
  __shared__ int odd_part[NW];
  static_assert(W * P * 4 >= kKeys * DH * 2, "a block's V rows fit");
  int h, idx;
  SeqTile t;
  packed_place(grid, h, idx);
  if (!find_tile<W>(a, idx, t)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lw = lane % W, slot = lane / W;
  // row of result register e: 16x16 slot*4 + e, 32x32 (e/4)*8 + slot*4 + e%4
  auto out_row = [&](int e) { return W == 16 ? slot * 4 + e : (e >> 2) * 8 + slot * 4 + (e & 3); };

  // this lane's row (rows past the sequence repeat its last one and are not stored)
  const int n_rows = t.len_q * a.group, r0 = t.tile * W;
  const int row = min(r0 + lw, n_rows - 1);
  const int seen = keys_seen(a, t, (int)a.by_group.quot(row));
  const int seen_lo = keys_seen(a, t, (int)a.by_group.quot(r0));  // the least and the greatest of the tile
  const int seen_hi = keys_seen(a, t, (int)a.by_group.quot(min(r0 + W - 1, n_rows - 1)));

  const bf16* kg = static_cast<const bf16*>(a.k) + (long)t.k0 * a.k_stride + (long)h * DH;
  const bf16* vg = static_cast<const bf16*>(a.v) + (long)t.k0 * a.v_stride + (long)h * DH;
  bf16x8 kf[KT][KK], vr[LV];
  auto load = [&](int n0) {
    if (n0 >= seen_hi) return;
    // uniform base (scalar) and 32-bit byte offsets; rows past the sequence repeat its last one
    const char* kb = reinterpret_cast<const char*>(kg + n0 * a.k_stride);
    const char* vb = reinterpret_cast<const char*>(vg + n0 * a.v_stride);
    const int last = t.len_k - 1 - n0;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const unsigned kr = (unsigned)min(kt * W + lw, last) * (unsigned)a.k_stride * 2 + slot * 16;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[kt][kk] = *reinterpret_cast<const bf16x8*>(kb + (kr + kk * 16 * SL));
    }
#pragma unroll
    for (int i = 0; i < LV; ++i) {
      const int f = i * 64 + lane;
      const unsigned vo = (unsigned)min(f / CPR, last) * (unsigned)a.v_stride * 2 + f % CPR * 16;
      vr[i] = *reinterpret_cast<const bf16x8*>(vb + vo);
    }
  };
  load(wave * kKeys);

  bf16x8 qf[KK];
  {
    const int i = (int)a.by_group.quot(row);
    const bf16* qr = static_cast<const bf16*>(a.q) + (t.q0 + i) * a.q_stride +
                     (long)(h * a.group + row - i * a.group) * DH + slot * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qr + kk * 8 * SL);
  }
  const float sl2e = a.scale * kLog2e;

  // V rows in LDS: chunk c of row r at slot c ^ f(r), so that the rows' writes
  // and the transpose reads (16 rows, 2 chunks; 32 rows' form 8 rows, 4 chunks) hit disjoint banks
  bf16* vl = reinterpret_cast<bf16*>(buf[wave]);
  auto swz = [](int r) {
    if (W == 16) return DH == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1;
    return DH == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
  };
  // V^T fragment of head-dim tile dt for k-step ks: the keys of the probabilities as they sit
  auto vfrag = [&](int dt, int ks) {
    const int r = slot % (W == 16 ? 4 : 2) * 4 + ((lane & 15) >> 2);
    const int col = dt * W + (W == 16 ? 0 : ((lane >> 4) & 1) * 16) + 4 * (lane & 3);
    const bf16* src = vl + (ks * 16 + r) * DH + (((col >> 3) ^ swz(r)) * 8) + (col & 7);
    const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src));
    const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src + (W == 16 ? 16 : 8) * DH));
    return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  Acc acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (Acc){};
  float m_run = -INFINITY, l_run = 0.f;
  // Where a row does not see a key its weight is 0, but 0 times an infinite
  // value is NaN. In blocks that some row does not see whole, values that are not
  // finite are left out of the products, and the merge adds them to the rows that see them.
  bool cut_odd = false;
  for (int n0 = wave * kKeys; n0 < seen_hi; n0 += NW * kKeys) {
    const bool cut = n0 + kKeys > seen_lo;  // some row does not see every key of the block
    if (cut) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < LV; ++i) odd |= odd8(vr[i]);
      if (__any(odd)) {
        cut_odd = true;
#pragma unroll
        for (int i = 0; i < LV; ++i) vr[i] = without_odd(vr[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < LV; ++i) {
      const int f = i * 64 + lane, r = f / CPR;
      *reinterpret_cast<bf16x8*>(vl + r * DH + ((f % CPR) ^ swz(r)) * 8) = vr[i];
    }
    Acc s[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) s[kt] = (Acc){};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) s[kt] = MfmaB<W>::mul(kf[kt][kk], qf[kk], s[kt]);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // the V rows are in LDS
    load(n0 + NW * kKeys);
    if (cut) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < NE; ++e)
          if (n0 + kt * W + out_row(e) >= seen) s[kt][e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < NE; ++e) mx = fmaxf(mx, s[kt][e]);
#pragma unroll
    for (int x = W; x < 64; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
    if (__any(mx > m_run)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run - m_new) * sl2e);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;  // no key or only -inf scores so far: weights 0
    bf16x4 pb[KT * NE / 4];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int g = 0; g < NE / 4; ++g) {
        f32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f((s[kt][g * 4 + e] - m_use) * sl2e);
          l_run += p[e];
        }
        pb[kt * (NE / 4) + g] = to_bf16x4(p);
      }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        acc[dt] = MfmaB<W>::mul(vfrag(dt, ks), __builtin_shufflevector(pb[2 * ks], pb[2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7), acc[dt]);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // read before the next block's rows
  }

  // merge: the waves' softmaxes, each rescaled to the common maximum.
  // acc[dt][e]: channel dt*W + out_row(e) of row lw
  float l_tot = l_run;
#pragma unroll
  for (int x = W; x < 64; x <<= 1) l_tot += __shfl_xor(l_tot, x);
  if (lane == 0) odd_part[wave] = cut_odd;
  if (slot == 0) {
    m_part[wave][lw] = m_run;
    l_part[wave][lw] = l_tot;
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < NE / 4; ++g)
      *reinterpret_cast<f32x4*>(&buf[wave][lw * P + dt * W + out_row(g * 4)]) =
          (f32x4){acc[dt][g * 4], acc[dt][g * 4 + 1], acc[dt][g * 4 + 2], acc[dt][g * 4 + 3]};
  __syncthreads();
  bool any_odd = false;
#pragma unroll
  for (int w = 0; w < NW; ++w) any_odd |= odd_part[w] != 0;
  for (int f = threadIdx.x; f < W * DH / 4; f += NW * 64) {
    const int r = f / (DH / 4), c = (f - r * (DH / 4)) * 4;
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
      const float wt = __builtin_amdgcn_exp2f((mw - m) * sl2e);
      l = fmaf(wt, l_part[w][r], l);
      sum += wt * *reinterpret_cast<const f32x4*>(&buf[w][r * P + c]);
    }
    const int i = (int)a.by_group.quot(R), hq = h * a.group + R - i * a.group;
    const long orow = (long)(t.q0 + i) * (a.kv_heads * a.group) + hq;
    sum *= l == 0.f ? 0.f : 1.f / l;
    if (any_odd && l != 0.f) add_odd(sum, vg + c, a.v_stride, max(seen_lo, 0) / kKeys * kKeys, keys_seen(a, t, i));
    *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + orow * DH + c) = to_bf16x4(sum);
    if (a.lse && c == 0)
      a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, __builtin_amdgcn_logf(l) * kLn2);
  }
}

template <int DH, int W, int NW>
hipError_t launch_small(const PackedArgs& a, hipStream_t s) {
  const PackedGrid g = packed_grid(a, W, DH * 2);
  if (g.groups < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_small_kernel<DH, W, NW>), dim3((unsigned)g.groups), dim3(NW * 64), 0, s, a, g);
  return hipGetLastError();
}

// Fitted to 499 launches of 1, 5 and 20 prompts of 1 to 4500 tokens, with and without 1000
// rows before them, 1 to 40 heads of either width: the least estimate takes 1.8% more
// than the fastest of the five on average, over 10% more in one launch of 19. Measured, us, in this
// order, no mask but for 20 prompts:
//   128-wide, 8 heads      1 prompt of 400 tokens   9.6    9.4   11.0   11.2   15.2
//                          1 of 1000               28.5   26.3   18.6   18.1   28.2
//                          1 of 4500                392    365    238    250    104
//                          20 of 25 to 77          14.4   10.5   12.2   13.1    8.6
//   64-wide, 32/8 heads    1 of 400                14.7   13.1   13.1   10.4    9.5
//                          1 of 1000               44.8   42.8   38.2   30.0   18.0
//                          20 of 25 to 77          19.4   11.2   19.7   12.0    8.4
constexpr PackedCost kCosts[2][5] = {{{16, 8, 2.5, 2.0, 0.132, 0.060},   // 64-wide heads
                                      {16, 4, 3.5, 0.87, 0.144, 0.050},
                                      {32, 8, 0.0, 4.8, 0.167, 0.067},
                                      {32, 4, 2.7, 2.3, 0.164, 0.207},
                                      {128, 4, 2.9, 3.0, 0.283, 0.357}},
                                     {{16, 8, 0.0, 5.0, 0.293, 0.136},   // 128-wide
                                      {16, 4, 3.0, 2.3, 0.274, 0.134},
                                      {32, 8, 0.0, 6.0, 0.351, 0.174},
                                      {32, 4, 0.0, 6.3, 0.351, 0.316},
                                      {256, 8, 0.0, 7.6, 0.719, 0.050}}};

template <int DH>
hipError_t launch_dh(const PackedArgs& a, hipStream_t s) {
  const PackedCost* c = packed_choice(a, kCosts[DH == 128]);
  if (!c) return hipErrorInvalidValue;
  if (c->rows >= 128) return launch_packed_attention_large(a, DH, s);
  if (c->rows == 32) return c->waves == 8 ? launch_small<DH, 32, 8>(a, s) : launch_small<DH, 32, 4>(a, s);
  return c->waves == 8 ? launch_small<DH, 16, 8>(a, s) : launch_small<DH, 16, 4>(a, s);
}

}  // namespace

PackedTile& packed_tile() {
  static thread_local PackedTile tile{0, 0};
  return tile;
}

hipError_t launch_packed_attention(const PackedArgs& a, bool bf16, int head_dim, hipStream_t s) {
  if (a.n_q <= 0 || a.n_seqs <= 0) return hipSuccess;
  if (!bf16) return launch_packed_attention_f32(a, head_dim, s);
  return head_dim == 64 ? launch_dh<64>(a, s) : launch_dh<128>(a, s);
}

}  // namespace hsa

void _hsa_packed_tile(int rows, int waves) { hsa::packed_tile() = {rows, waves}; }
