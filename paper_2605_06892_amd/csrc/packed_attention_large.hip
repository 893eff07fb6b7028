// bf16 attention of packed sequences: 256 rows of one 128-wide key/value head per
// workgroup, 128 of a 64-wide one (rows are (query, head of the group) pairs, see packed.h).
//
// 8 or 4 waves of 32 rows. K/V tiles of 96 keys go global -> LDS directly, three tiles deep
// (144 or 72 KB of LDS), issued two tiles ahead by one wave per SIMD,
// one barrier per tile. LDS rows are unpadded, their 16-byte chunks permuted by an XOR with
// a function of the row, so that the K fragment reads (16 rows, one chunk) and the V
// transpose reads (4 rows, 4 chunks) hit disjoint banks. Per 32-key block and wave:
//   S^T = K Q^T - m   v_mfma_f32_32x32x16_bf16, K rows the A operand from LDS,
//                   the wave's Q fragments resident as the B operand. The
//                   accumulator is seeded with -m, the row's reference maximum of
//                   the unscaled products, so that what the exponential gets is
//                   exact however large the products are.
//   softmax         exp2(scale log2(e) s), a running sum and the bf16 pack per
//                   score. m is set from the first keys a row sees and raised
//                   only when some weight of a block exceeds 2^16.
//   O^T += V^T P^T  the weights, rounded to bf16, are the B operand as they sit
//                   in the score accumulators; the V^T operand comes from
//                   ds_read_b64_tr_b16.
// The S^T MFMAs of block b+1 are issued next to the exponentials of block b.
// A wave leaves out the blocks that none of its rows sees.
#include "packed.h"

#include <type_traits>

namespace hsa {
namespace {

constexpr int BKV = 96;                 // keys per LDS tile (three 32-key blocks)
constexpr int NBUF = 3;                 // LDS tiles in flight
constexpr float kSlowSum = 65536.0f;    // 2^16: raise the reference maximum

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_cvoid;

// s_waitcnt immediate for "vector memory counter <= n", other counters free
constexpr int waitcnt_vm(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }

// chunk permutation of key row r inside a tile
template <int DH>
__device__ __forceinline__ int swz_k(int r) {
  return DH == 128 ? (((r & 3) << 2) | ((r >> 2) & 3)) : ((r >> 1) & 7);
}
template <int DH>
__device__ __forceinline__ int swz_v(int r) {
  return DH == 128 ? ((r & 3) << 2) : (((r >> 1) & 1) << 2);
}

// Waves of a workgroup. At 64-wide heads LDS holds two workgroups of 4 waves per CU, which start and
// end apart from each other: as fast as one of 8 on long prompts (32/8 heads, 8000 causal
// tokens 281 and 277 us), faster where tiles are few (1000 tokens 17 and 21). At 128 it holds one, and
// a wave alone on its SIMD takes as long for a block as each of two: 1000 tokens 31 and 28 us, 3000
// 138 and 81.
template <int DH>
constexpr int waves = DH == 64 ? 4 : 8;

template <int DH>
__global__ __launch_bounds__(waves<DH> * 64, 2) void packed_large_kernel(PackedArgs a, PackedGrid grid) {
  constexpr int NW = waves<DH>, BQ = NW * 32;
  constexpr int CPR = DH / 8;        // 16-byte chunks per key row
  constexpr int RPS = 64 / CPR;      // rows per 1 KB LDS segment
  constexpr int SEGS = BKV / RPS;    // segments per tile
  constexpr int DT = DH / 32;        // 32-wide head-dim tiles of O^T
  constexpr int KK = DH / 16;        // k-steps of S^T
  // one array per buffer: with compile-time buffer indices the compiler can
  // tell the asynchronous tile loads from the LDS reads of other buffers
  __shared__ __attribute__((aligned(16))) bf16 K0[BKV * DH], K1[BKV * DH], K2[BKV * DH];
  __shared__ __attribute__((aligned(16))) bf16 V0[BKV * DH], V1[BKV * DH], V2[BKV * DH];
  auto kbuf = [&](auto b) -> bf16* {
    constexpr int B = decltype(b)::value;
    if constexpr (B == 0) return K0; else if constexpr (B == 1) return K1; else return K2;
  };
  auto vbuf = [&](auto b) -> bf16* {
    constexpr int B = decltype(b)::value;
    if constexpr (B == 0) return V0; else if constexpr (B == 1) return V1; else return V2;
  };

  __shared__ int odd_flag;  // a value was taken out, see take_odd
  int h, idx;
  SeqTile t;
  packed_place(grid, h, idx);
  if (!find_tile<BQ>(a, idx, t)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // uniform: scalar
  const int l32 = lane & 31, hi = lane >> 5;
  const float sl2e = a.scale * kLog2e;

  // this lane's row (rows past the sequence repeat its last one and are not stored)
  const int n_rows = t.len_q * a.group, r0 = t.tile * BQ, rw = r0 + wave * 32;
  const int row = min(rw + l32, n_rows - 1), qi = (int)a.by_group.quot(row);
  const int seen = keys_seen(a, t, qi);
  // keys up to which some, and all, rows of the wave see, and the workgroup's last one
  const int seen_hi = rw < n_rows ? keys_seen(a, t, (int)a.by_group.quot(min(rw + 31, n_rows - 1))) : 0;
  const int seen_lo = keys_seen(a, t, (int)a.by_group.quot(min(rw, n_rows - 1)));
  const int kv_end = keys_seen(a, t, (int)a.by_group.quot(min(r0 + BQ - 1, n_rows - 1)));

  // Q fragments: lane holds Q[row l32][kk*16 + hi*8 + 0..7]. Half rows are loaded,
  // a line at a time, and go through a part of the tile buffer that is loaded
  // last (straight into this layout, 32 bytes of a row at a time, they took 1.2 us longer).
  constexpr int QC = CPR / 2, QL = 32 * QC / 64;  // chunks of a half row, loads of the wave's half rows
  bf16x8 qf[KK], qx[2][QL];
  const int q_row = lane / QC, q_chunk = lane % QC;
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < QL; ++i) {
      const int R = min(rw + i * (64 / QC) + q_row, n_rows - 1), j = (int)a.by_group.quot(R);
      qx[half][i] = *reinterpret_cast<const bf16x8*>(
          static_cast<const bf16*>(a.q) + (long)(t.q0 + j) * a.q_stride +
          (long)(h * a.group + R - j * a.group) * DH + (half * QC + q_chunk) * 8);
    }

  // this lane's part of a tile load: segment seg = i*LW + wave, row seg*RPS + lane/CPR,
  // LDS slot lane%CPR holding global chunk slot ^ f(row). Loads come from waves
  // 0..3 only, one per SIMD: a wave stalls while its loads issue, and the other
  // wave of its SIMD, where there is one, keeps the matrix pipe busy meanwhile.
  const bf16* kg = static_cast<const bf16*>(a.k) + (long)t.k0 * a.k_stride + (long)h * DH;
  const bf16* vg = static_cast<const bf16*>(a.v) + (long)t.k0 * a.v_stride + (long)h * DH;
  constexpr int LW = 4;                 // loader waves
  constexpr int LL = SEGS / LW;         // segment loads per loader wave per tensor
  constexpr int RSTEP = RPS * LW;       // tile rows between a loader's segments
  static_assert(LL * LW == SEGS, "loader waves must cover the tile");
  static_assert(RSTEP % 16 == 0, "one chunk permutation for all of a loader's rows");
  const int lr = wave * RPS + lane / CPR;
  const int kch = ((lane % CPR) ^ swz_k<DH>(lr)) * 8, vch = ((lane % CPR) ^ swz_v<DH>(lr)) * 8;
  const unsigned k_lane = (unsigned)(lr * (int)a.k_stride + kch) * 2;  // bytes from the tile's first row
  const unsigned v_lane = (unsigned)(lr * (int)a.v_stride + vch) * 2;
  auto issue_tile = [&](auto buf, int kv0) {
    if (wave >= LW) return;
    bf16* kd = kbuf(buf) + wave * 512;
    bf16* vd = vbuf(buf) + wave * 512;
    if (kv0 + BKV <= t.len_k) {
      // uniform tile base (scalar) + the lane's byte offset
      const char* ks = reinterpret_cast<const char*>(kg + kv0 * a.k_stride);
      const char* vs = reinterpret_cast<const char*>(vg + kv0 * a.v_stride);
#pragma unroll
      for (int i = 0; i < LL; ++i) {
        __builtin_amdgcn_global_load_lds((global_cvoid*)(ks + i * RSTEP * a.k_stride * 2 + k_lane),
                                         (lds_void*)(kd + i * LW * 512), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_cvoid*)(vs + i * RSTEP * a.v_stride * 2 + v_lane),
                                         (lds_void*)(vd + i * LW * 512), 16, 0, 0);
      }
    } else {  // the sequence ends in this tile: rows past it repeat its last one
#pragma unroll
      for (int i = 0; i < LL; ++i) {
        const long n = min(kv0 + lr + i * RSTEP, t.len_k - 1);
        __builtin_amdgcn_global_load_lds((global_cvoid*)(kg + n * a.k_stride + kch), (lds_void*)(kd + i * LW * 512), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_cvoid*)(vg + n * a.v_stride + vch), (lds_void*)(vd + i * LW * 512), 16, 0, 0);
      }
    }
  };

  // LDS element offsets this lane reads, relative to a 32-key block
  int koff[KK];  // K fragment kk: row l32, chunk kk*2 + hi
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) koff[kk] = l32 * DH + (((kk * 2 + hi) ^ swz_k<DH>(l32)) * 8);
  int voff[DT];  // V transpose read, head-dim tile dt: row hi*4 + k, channel dt*32 + 16g + 4(lane&3)
  {
    const int k4 = (lane & 15) >> 2, g = (lane >> 4) & 1;
    const int r = hi * 4 + k4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int col = dt * 32 + 16 * g + 4 * (lane & 3);
      voff[dt] = r * DH + (((col >> 3) ^ swz_v<DH>(r)) * 8) + (col & 7);
    }
  }

  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x16){};
  f32x16 negm = (f32x16){};  // every element -m_ref: the seed of the score accumulators
  float m_ref = 0.f, l_run = 0.f;
  bool have_ref = false;     // whether this row has seen a score above -infinity
  constexpr int KP = KK < 4 ? KK : 4;  // K fragments read one step ahead, during the previous block's PV
  bf16x8 kpre[KP];
  auto kfrag = [&](auto buf, int kb, int kk) {
    return *reinterpret_cast<const bf16x8*>(kbuf(buf) + kb * DH + koff[kk]);
  };

  // S^T of the 32-key block starting at row kb of tile buffer buf
  auto scores = [&](auto buf, int kb, f32x16& s) {
    const bf16* base = kbuf(buf) + kb * DH;
    bf16x8 kf[KK];
#pragma unroll
    for (int kk = 0; kk < KP; ++kk) kf[kk] = kpre[kk];
#pragma unroll
    for (int kk = KP; kk < KK; ++kk) kf[kk] = *reinterpret_cast<const bf16x8*>(base + koff[kk]);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], negm, 0, 0, 0);
#pragma unroll
    for (int kk = 1; kk < KK; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], s, 0, 0, 0);
  };

  // One pipeline step: S^T of the next block, softmax of the current block
  // (keys key0 .. key0+31, V rows vb .. of buffer buf), PV. The next block's
  // scores always come from a valid LDS address, so that they share a scheduling
  // region with the softmax; after the last block they are unused.
  auto step = [&](f32x16& s_cur, f32x16& s_nxt, auto nbuf, int nkb, auto buf, int vb, int key0,
                  auto nnbuf, int nnkb) {
    if (key0 + 32 > seen_lo) {  // some row does not see every key of the block
      const int kbase = key0 + hi * 4;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (kbase + (e >> 2) * 8 + (e & 3) >= seen) s_cur[e] = -INFINITY;
    }
    scores(nbuf, nkb, s_nxt);
    const bf16* vbase = vbuf(buf) + vb * DH;
    constexpr int NV = 1;  // head-dim tiles whose V fragments are read before the softmax
    bf16x8 vfa[NV][2];
#pragma unroll
    for (int dt = 0; dt < NV; ++dt)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16* src = vbase + ks * 16 * DH + voff[dt];
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src));
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src + 8 * DH));
        vfa[dt][ks] = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(s_cur[e] * sl2e);
    auto sum = [&] {
      return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])) +
             (((p[8] + p[9]) + (p[10] + p[11])) + ((p[12] + p[13]) + (p[14] + p[15])));
    };
    float ls = sum();
    bool raise = !have_ref || !(ls <= kSlowSum);
    if (__any(raise)) {
      // set or raise the reference maximum of the rows that need it, rescale what they accumulated
      raise |= (bool)__shfl_xor((int)raise, 32);        // the row's other half
      float mx = s_cur[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s_cur[e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));               // block max relative to m_ref
      // amount to raise m_ref by; a row without a score yet keeps it
      const float up = !raise || mx == -INFINITY ? 0.f : (have_ref ? fmaxf(mx, 0.f) : mx);
      const float alpha = have_ref ? __builtin_amdgcn_exp2f(-up * sl2e) : 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f((s_cur[e] - up) * sl2e);
      ls = sum();
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      m_ref += up;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        negm[e] = -m_ref;
        s_nxt[e] -= up;  // the next block's scores were seeded with the old reference
      }
      have_ref = have_ref || mx > -INFINITY;
    }
    l_run += ls;
    bf16x8 pf[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x4 lo = {p[8 * half + 0], p[8 * half + 1], p[8 * half + 2], p[8 * half + 3]};
      f32x4 up = {p[8 * half + 4], p[8 * half + 5], p[8 * half + 6], p[8 * half + 7]};
      pf[half] = __builtin_shufflevector(to_bf16x4(lo), to_bf16x4(up), 0, 1, 2, 3, 4, 5, 6, 7);
    }
#pragma unroll
    for (int kk = 0; kk < KP; ++kk) kpre[kk] = kfrag(nnbuf, nnkb, kk);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        bf16x8 vf;
        if (dt < NV) {
          vf = vfa[dt][ks];
        } else {
          const bf16* src = vbase + ks * 16 * DH + voff[dt];
          const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src));
          const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(src + 8 * DH));
          vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[ks], acc[dt], 0, 0, 0);
      }
    }
  };

  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  using B2 = std::integral_constant<int, 2>;
  const int n_tiles = kv_end > 0 ? (kv_end + BKV - 1) / BKV : 0;
  const int n_full = max(keys_seen(a, t, (int)a.by_group.quot(r0)), 0) / BKV;  // tiles that every row sees whole
  // Where a row does not see a key its weight is 0, but 0 times an infinite
  // value is NaN. In the tiles that some row does not see whole, values that are not
  // finite are taken out by the wave that loaded them, and added to the rows that
  // see them at the end.
  auto take_odd = [&](auto buf) {
    if (wave >= LW) return;
    bf16* v = vbuf(buf) + wave * 512 + lane * 8;  // what this wave has loaded
#pragma unroll
    for (int i = 0; i < LL; ++i) {
      bf16x8* at = reinterpret_cast<bf16x8*>(v + i * LW * 512);
      const bf16x8 x = *at;
      if (odd8(x)) {
        *at = without_odd(x);
        odd_flag = 1;
      }
    }
  };
  if (threadIdx.x == 0) odd_flag = 0;
  __syncthreads();
  if (n_tiles > 0) {
    issue_tile(B0{}, 0);
    if (n_tiles > 1) issue_tile(B1{}, BKV);
    {
      constexpr int EACH = 32 * QC * 8, PER = BKV * DH / EACH;  // values of a wave, waves to a buffer
      static_assert(2 * PER >= NW, "two buffers hold the waves' half rows");
      bf16* ql = (wave < PER ? K2 : V2) + wave % PER * EACH;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < QL; ++i) {
          const int r = i * (64 / QC) + q_row;
          *reinterpret_cast<bf16x8*>(ql + (r * QC + (q_chunk ^ (r & (QC - 1)))) * 8) = qx[half][i];
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
        for (int kk = 0; kk < KK / 2; ++kk)
          qf[half * (KK / 2) + kk] = *reinterpret_cast<const bf16x8*>(ql + (l32 * QC + ((kk * 2 + hi) ^ (l32 & (QC - 1)))) * 8);
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    if (n_full == 0) take_odd(B0{});
    __syncthreads();
    f32x16 sa, sb;
#pragma unroll
    for (int kk = 0; kk < KP; ++kk) kpre[kk] = kfrag(B0{}, 0, kk);
    scores(B0{}, 0, sa);
#pragma unroll
    for (int kk = 0; kk < KP; ++kk) kpre[kk] = kfrag(B0{}, 32, kk);
    // Tile it lives in buffer it % 3; the loop is unrolled by 3 so that every
    // buffer index is a compile-time constant. s0 holds the scores of the tile's
    // block 0 on entry; the three steps alternate the two score registers, so the
    // next tile starts from s1.
    auto tile = [&](auto buf, auto nxt, auto nn, int it, f32x16& s0, f32x16& s1) {
      const int kv0 = it * BKV;
      if (kv0 < seen_hi) step(s0, s1, buf, 32, buf, 0, kv0, buf, 64);
      // tile it+1 (issued one tile ago) has landed; after this barrier every
      // wave is done with tile it-1, whose buffer receives tile it+2
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
      if (it + 1 >= n_full && it + 1 < n_tiles) take_odd(nxt);  // the next tile has a mask
      __syncthreads();
      if (it + 2 < n_tiles) issue_tile(nn, kv0 + 2 * BKV);
      if (kv0 + 32 < seen_hi) step(s1, s0, buf, 64, buf, 32, kv0 + 32, nxt, 0);
      if (kv0 + 64 < seen_hi) step(s0, s1, nxt, 0, buf, 64, kv0 + 64, nxt, 32);
    };
    for (int it = 0; it < n_tiles; it += NBUF) {
      tile(B0{}, B1{}, B2{}, it, sa, sb);
      if (it + 1 < n_tiles) tile(B1{}, B2{}, B0{}, it + 1, sb, sa);
      if (it + 2 < n_tiles) tile(B2{}, B0{}, B1{}, it + 2, sa, sb);
      const f32x16 x = sa;  // three tiles of three steps: the roles swap
      sa = sb;
      sb = x;
    }
  }
  const bool cut_odd = odd_flag != 0;

  // acc[dt][e]: channel dt*32 + (e/4)*8 + hi*4 + e%4 of row l32
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  const bool none = l_tot == 0.f;  // no key, or no finite score: zeros, also where acc holds 0 * infinity
  const float inv = 1.f / l_tot;
  // The rows go through LDS, so that whole lines of them are stored (8 bytes of
  // a row at a time took 2 us longer).
  __syncthreads();  // every wave is done with the tiles
  constexpr int PER = BKV / 32;  // waves to a buffer
  bf16* ol = (wave < PER ? K0 : (wave < 2 * PER ? K1 : K2)) + wave % PER * (32 * DH);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = dt * 32 + g * 8 + hi * 4;
      f32x4 v = {acc[dt][4 * g + 0] * inv, acc[dt][4 * g + 1] * inv, acc[dt][4 * g + 2] * inv,
                 acc[dt][4 * g + 3] * inv};
      if (none) v = (f32x4){};
      else if (cut_odd) add_odd(v, vg + c, a.v_stride, n_full * BKV, seen);
      *reinterpret_cast<bf16x4*>(ol + l32 * DH + (((dt * 4 + g) ^ (l32 & (CPR - 1))) * 8) + hi * 4) = to_bf16x4(v);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  auto head_row = [&](int R) -> long {  // of o and lse
    const int i = (int)a.by_group.quot(R);
    return (long)(t.q0 + i) * (a.kv_heads * a.group) + h * a.group + (R - i * a.group);
  };
#pragma unroll
  for (int i = 0; i < 32 * CPR / 64; ++i) {
    const int r = (i * 64 + lane) / CPR, c = lane % CPR;
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(ol + r * DH + ((c ^ (r & (CPR - 1))) * 8));
    if (rw + r < n_rows) *reinterpret_cast<bf16x8*>(static_cast<bf16*>(a.o) + head_row(rw + r) * DH + c * 8) = x;
  }
  if (a.lse && hi == 0 && rw + l32 < n_rows)
    a.lse[head_row(rw + l32)] = none ? -INFINITY : fmaf(m_ref, a.scale, __builtin_amdgcn_logf(l_tot) * kLn2);
}

template <int DH>
hipError_t launch(const PackedArgs& a, hipStream_t s) {
  const PackedGrid g = packed_grid(a, waves<DH> * 32, DH * 2);
  if (g.groups < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_large_kernel<DH>), dim3((unsigned)g.groups), dim3(waves<DH> * 64), 0, s, a, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_attention_large(const PackedArgs& a, int head_dim, hipStream_t s) {
  return head_dim == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace hsa
