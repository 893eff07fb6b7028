// bf16 attention of packed sequences with grouped heads, causal or not.
//
//   o_i = sum_j softmax_j(scale <q_i, k_j>) v_j over the keys that query i sees
//
// Small tiles: 16 rows (see packed.h) of one key/value head per workgroup, whose 8 waves
// split the keys (wave w takes the 32-key blocks w, w+8, ...) and merge their
// softmaxes in LDS. Per block of a wave: S^T = K Q^T by
// v_mfma_f32_16x16x32_bf16, K rows straight from global memory in the A
// operand's layout (lane: key l16, channels grp*8 ..); each lane holds 8 scores
// of ONE row (keys kt*16 + grp*4 + e), which are the B operand of O^T += V^T P^T
// as they sit (slot grp*8 + kt*4 + e). V rows go through the wave's LDS region
// for the transpose read. Both are loaded one block ahead.
//
// Scores are exact products of the bf16 inputs, and the scale follows the
// subtraction of the running maximum in fp32. Rounded to bf16 are the probabilities
// (the sum takes them before that) and the output.
#include "packed.h"

namespace hsa {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// true if one of 8 bf16 values is not finite
__device__ __forceinline__ bool odd8(bf16x8 x) {
  const u32x4 u = __builtin_bit_cast(u32x4, x);
  unsigned r = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) r |= (u[j] & 0x7f807f80u) + 0x00800080u;
  return r & 0x80008000u;
}

// the finite ones of 8 bf16 values, and zeros for the others
__device__ __forceinline__ bf16x8 without_odd(bf16x8 x) {
  u32x4 u = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned hit = ((u[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // top bit of each half that is not
    u[j] &= ~((hit >> 15) * 0xffffu);
  }
  return __builtin_bit_cast(bf16x8, u);
}

// adds to 4 channels of a row the values of keys from .. end-1 that are not finite
__device__ __forceinline__ void add_odd(f32x4& sum, const bf16* v, long stride, int from, int end) {
  for (int n = from; n < end; ++n)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float x = (float)v[n * stride + u];
      if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) sum[u] += x;
    }
}

constexpr int kSmallWaves = 8, kSmallRows = 16;

template <int DH>
__global__ __launch_bounds__(kSmallWaves * 64) void packed_small_kernel(PackedArgs a, PackedGrid grid) {
  constexpr int KK = DH / 32;              // k-steps of S^T
  constexpr int DT = DH / 16;              // 16-wide head-dim tiles of O^T
  constexpr int CPR = DH / 8;              // 16-byte chunks per row
  constexpr int LV = 32 * CPR / 64;        // V loads per lane and block
  constexpr int P = DH + 4;                // padded row of the merge buffer, floats
  __shared__ __attribute__((aligned(16))) float buf[kSmallWaves][kSmallRows * P];  // V rows, then the merge
  __shared__ float m_part[kSmallWaves][kSmallRows], l_part[kSmallWaves][kSmallRows];
  __shared__ int odd_part[kSmallWaves];
  static_assert(kSmallRows * P * 4 >= 32 * DH * 2, "a block's V rows fit");
  int h, idx;
  SeqTile t;
  packed_place(grid, a.kv_heads, h, idx);
  if (!find_tile(a, idx, kSmallRows, t)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, grp = lane >> 4;

  // this lane's row (rows past the sequence repeat its last one and are not stored)
  const int n_rows = t.len_q * a.group, r0 = t.tile * kSmallRows;
  const int row = min(r0 + l16, n_rows - 1);
  const int seen = keys_seen(a, t, row / a.group);
  const int seen_lo = keys_seen(a, t, r0 / a.group);  // the least and the greatest of the tile
  const int seen_hi = keys_seen(a, t, min(r0 + kSmallRows - 1, n_rows - 1) / a.group);

  const bf16* kg = static_cast<const bf16*>(a.k) + (long)t.k0 * a.k_stride + (long)h * DH;
  const bf16* vg = static_cast<const bf16*>(a.v) + (long)t.k0 * a.v_stride + (long)h * DH;
  bf16x8 kf[2][KK], vr[LV];
  auto load = [&](int n0) {
    if (n0 >= seen_hi) return;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {  // rows past the sequence repeat its last one
      const bf16* kr = kg + min(n0 + kt * 16 + l16, t.len_k - 1) * a.k_stride + grp * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[kt][kk] = *reinterpret_cast<const bf16x8*>(kr + kk * 32);
    }
#pragma unroll
    for (int i = 0; i < LV; ++i) {
      const int f = i * 64 + lane;
      vr[i] = *reinterpret_cast<const bf16x8*>(vg + min(n0 + f / CPR, t.len_k - 1) * a.v_stride + f % CPR * 8);
    }
  };
  load(wave * 32);

  bf16x8 qf[KK];
  {
    const int i = row / a.group;
    const bf16* qr = static_cast<const bf16*>(a.q) + (t.q0 + i) * a.q_stride +
                     (long)(h * a.group + row - i * a.group) * DH + grp * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qr + kk * 32);
  }
  const float sl2e = a.scale * kLog2e;

  // V rows in LDS: chunk c of row r at slot c ^ f(r), so that the rows' writes
  // and the transpose reads (16 rows, 2 chunks) hit disjoint banks
  bf16* vl = reinterpret_cast<bf16*>(buf[wave]);
  auto swz = [](int r) { return DH == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1; };
  auto vfrag = [&](int dt) {
    const int r = grp * 4 + (l16 >> 2), col = dt * 16 + 4 * (lane & 3);
    const bf16* src = vl + r * DH + (((col >> 3) ^ swz(r)) * 8) + (col & 7);
    const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src));
    const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src + 16 * DH));
    return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){};
  float m_run = -INFINITY, l_run = 0.f;
  // Where a row does not see a key its weight is 0, but 0 times an infinite
  // value is NaN. In blocks that some row does not see whole, values that are not
  // finite are left out of the products, and the merge adds them to the rows that see them.
  bool cut_odd = false;
  for (int n0 = wave * 32; n0 < seen_hi; n0 += kSmallWaves * 32) {
    const bool cut = n0 + 32 > seen_lo;  // some row does not see every key of the block
    if (cut) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < LV; ++i) odd |= odd8(vr[i]);
      if (__any(odd)) {  // see cut_odd
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
    f32x4 s[2] = {};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
        s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kt][kk], qf[kk], s[kt], 0, 0, 0);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // the V rows are in LDS
    load(n0 + kSmallWaves * 32);
    if (cut) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n0 + kt * 16 + grp * 4 + e >= seen) s[kt][e] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                     fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__any(mx > m_run)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run - m_new) * sl2e);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;  // no key or only -inf scores so far: weights 0
    f32x4 p[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[kt][e] = __builtin_amdgcn_exp2f((s[kt][e] - m_use) * sl2e);
        l_run += p[kt][e];
      }
    const bf16x8 pf = __builtin_shufflevector(to_bf16x4(p[0]), to_bf16x4(p[1]), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vfrag(dt), pf, acc[dt], 0, 0, 0);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // read before the next block's rows
  }

  // merge: the waves' softmaxes, each rescaled to the common maximum.
  // acc[dt][e]: channel dt*16 + grp*4 + e of row l16
  float l_tot = l_run + __shfl_xor(l_run, 16);
  l_tot += __shfl_xor(l_tot, 32);
  if (lane == 0) odd_part[wave] = cut_odd;
  if (grp == 0) {
    m_part[wave][l16] = m_run;
    l_part[wave][l16] = l_tot;
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<f32x4*>(&buf[wave][l16 * P + dt * 16 + grp * 4]) = acc[dt];
  __syncthreads();
  bool any_odd = false;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) any_odd |= odd_part[w] != 0;
  for (int f = threadIdx.x; f < kSmallRows * DH / 4; f += kSmallWaves * 64) {
    const int r = f / (DH / 4), c = (f - r * (DH / 4)) * 4;
    const int R = r0 + r;
    if (R >= n_rows) continue;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) m = fmaxf(m, m_part[w][r]);
    f32x4 sum = {};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) {
      const float mw = m_part[w][r];
      if (mw == -INFINITY && l_part[w][r] == 0.f) continue;  // no key, or no finite score
      const float wt = __builtin_amdgcn_exp2f((mw - m) * sl2e);
      l = fmaf(wt, l_part[w][r], l);
      sum += wt * *reinterpret_cast<const f32x4*>(&buf[w][r * P + c]);
    }
    const int i = R / a.group, hq = h * a.group + R - i * a.group;
    const long orow = (long)(t.q0 + i) * (a.kv_heads * a.group) + hq;
    sum *= l == 0.f ? 0.f : 1.f / l;
    if (any_odd) add_odd(sum, vg + c, a.v_stride, max(seen_lo, 0) / 32 * 32, keys_seen(a, t, i));
    *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + orow * DH + c) = to_bf16x4(sum);
    if (a.lse && c == 0)
      a.lse[orow] = l == 0.f ? -INFINITY : fmaf(m, a.scale, __builtin_amdgcn_logf(l) * kLn2);
  }
}

template <int DH>
hipError_t launch_small(const PackedArgs& a, hipStream_t s) {
  const PackedGrid g = packed_grid(a.n_q, a.n_seqs, a.kv_heads, a.group, kSmallRows);
  if (g.groups < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_small_kernel<DH>), dim3((unsigned)g.groups), dim3(kSmallWaves * 64), 0, s, a, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_attention(const PackedArgs& a, bool bf16, int head_dim, hipStream_t s) {
  if (a.n_q <= 0 || a.n_seqs <= 0) return hipSuccess;
  if (!bf16) return launch_packed_attention_f32(a, head_dim, s);
  return head_dim == 64 ? launch_small<64>(a, s) : launch_small<128>(a, s);
}

}  // namespace hsa
