// Attention of one query per sequence over a paged cache of bf16, fp32 or e4m3
// rows, with grouped heads. It reads every cached row of a key/value head once for
// all the query heads of its group, and that reading bounds it.
//
// Work split. An item is (sequence, key/value head, 16 query heads of its group). Where no
// sequence can be longer than whole_len() rows, an item is a workgroup of 8 waves. Longer
// ones come in tiles of 128 rows: all tiles of all items, in order, are dealt to the
// workgroups (of 4 waves) in equal runs, so that a batch of very different lengths
// loads the CUs evenly and one long sequence is spread over all of them. A run that holds a
// whole item writes its output; the first and the last item of a run may be parts, which
// go to the workspace (unnormalized output, maximum and sum of the softmax) and are
// joined by a second kernel. Every run works out from the lengths where it begins, and leaves
// a note of the item that it begins and does not end: no atomics, no state between calls.
//
// In a workgroup, each wave takes every NW-th block of the item's rows, 32 keys
// of bf16 or e4m3 rows (16 with fp32 queries), one block loaded ahead (its page one more
// ahead: loads return in order, and a wait for a page loaded behind a block would be
// a wait for that block), with its own running softmax; they are merged in LDS
// at the end of an item. The 16 query heads are one column tile of the matrix instructions, in
// S^T = K Q^T and, with the probabilities as they sit in the score registers, in
// O^T += V^T P^T.
//   bf16   16x16x32: K rows in the A operand's layout straight from global
//          memory, V rows through LDS for the transpose read. e4m3 rows become bf16 first,
//          without a rounding (4 significant bits and a power of two).
//   fp32   16x16x4: K and V rows both in their operand's layout.
// Probabilities are rounded to bf16 in the bf16 form; the sums take them before that.
#include "paged.h"

namespace hsa {
namespace {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kSplitWaves = 4, kWholeWaves = 8;

// One item, or the rows key0 .. key1-1 of one, by NW waves.
template <bool F32, bool E4M3, int DH, bool ALIGNED, int NW>
struct Attend {
  static constexpr int BK = F32 ? 16 : 32;        // keys per block
  static constexpr int KT = BK / 16;              // key tiles of a block
  static constexpr int DT = DH / 16;              // channel tiles of O^T
  static constexpr int P = DH + 4;                // padded row of the merge buffer, floats
  static constexpr int ES = E4M3 ? 1 : (F32 ? 4 : 2);
  static constexpr int CB = 16;                   // bytes of a load
  static constexpr int CE = CB / ES;              // values of a load
  static constexpr int KL = DH / CE / 4;          // K loads per lane and key tile (its 4 slots share a row)
  // V: bf16 form, whole rows over the wave; fp32 form, DT consecutive channels of the 4 keys of a slot
  static constexpr int VR = F32 ? 4 : BK * DH / CE / 64;
  static constexpr int VB = F32 ? DT * ES : CB;   // bytes of one V read
  static constexpr int CPR = DH / CE;             // loads per row
  static constexpr unsigned kAll = BK == 32 ? ~0u : 0xffffu;
  struct VLoad { unsigned char b[VB]; };
  struct Shared {
    float buf[NW][kRows * P];  // V rows, then the merge
    float m_part[NW][kRows], l_part[NW][kRows];
  };
  static_assert(F32 || kRows * P * 4 >= BK * DH * 2, "a block's V rows fit");

  // The bf16 form loads whole rows of V, which nothing reads again: past the caches. K, whose rows
  // several loads share, stays (four sequences of 30011 to 131072: 226 us, V past the
  // caches 216, both 238).
  static __device__ __forceinline__ void load_v(VLoad& v, const char* p) {
    if constexpr (F32) {
      __builtin_memcpy(&v, p, VB);
    } else {
      const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
      __builtin_memcpy(&v, &x, VB);
    }
  }

  // 4 keys of 2 codes each as bf16, times a power of two: exact
  static __device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi, float scale) {
    bf16x8 y;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u ? hi : lo, scale, false);
      const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u ? hi : lo, scale, true);
      y[4 * u] = a[0], y[4 * u + 1] = a[1], y[4 * u + 2] = b[0], y[4 * u + 3] = b[1];
    }
    return y;
  }

  // s, h, g0 (first query head of the group), key0 and key1 are uniform. part:
  // where the unnormalized result goes, NULL for the output itself.
  static __device__ __forceinline__ void run(const PagedArgs& a, const Plan& plan, Shared& sh, int s, int h, int g0,
                                             int key0, int key1, Part<DH>* part) {
    const int lane = threadIdx.x & 63;
    const int wave = uniform(threadIdx.x >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const unsigned row_bytes = (unsigned)(a.kv_heads * DH) * ES;
    const float sl2e = a.scale * kLog2e;
    const int32_t* pages = a.page_table + (long)s * a.max_pages;
    bf16* vl = reinterpret_cast<bf16*>(sh.buf[wave]);
    // V rows in LDS: chunk c of row r at slot c ^ f(r), so that the rows' writes and
    // the transpose reads (16 rows, 2 chunks) spread over the banks
    auto swz = [](int r) { return DH == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1; };

    // one block ahead: its rows (as held), exponents, and which of its keys exist;
    // two blocks ahead: the page of this lane's key (lane % BK; ALIGNED: of all keys)
    u32x4 kr[KT][KL];
    VLoad vr[VR];
    int ke[KT], ve[VR];
    unsigned mask = 0;
    int page = -1;
    auto load_page = [&](int n0) {
      const int t = n0 + (ALIGNED ? 0 : lane % BK);
      page = -1;
      if (t < key1) page = pages[plan.page.quot(t)];
    };
    auto v_key = [&](int i) { return F32 ? grp * 4 + i : (i * 64 + lane) / CPR; };
    // byte offsets of this lane's loads in a block's rows, where those are consecutive
    const unsigned k_off = l16 * row_bytes + grp * CB;
    const unsigned v_off = F32 ? (unsigned)grp * 4 * row_bytes + l16 * VB : (lane / CPR) * row_bytes + lane % CPR * CB;
    auto load = [&](int n0) {
      if (n0 >= key1) return;
      const int t = n0 + (ALIGNED ? 0 : lane % BK);
      const bool ok = t < key1 && page >= 0 && page < a.n_pages;
      int first = ok ? page * a.page_size + (t - (int)plan.page.quot(t) * a.page_size) : 0;
      mask = ALIGNED ? (ok ? (key1 - n0 >= BK ? kAll : (1u << (key1 - n0)) - 1) : 0u) : (unsigned)__ballot(ok) & kAll;
      if constexpr (ALIGNED) {  // a block lies in one page: rows first ..
        first = uniform(first);
        load_page(n0 + NW * BK);
        const char* kb = static_cast<const char*>(a.k) + (long)first * row_bytes + h * (DH * ES);
        const char* vb = static_cast<const char*>(a.v) + (long)first * row_bytes + h * (DH * ES);
        const int8_t* keb = a.k_exp + (long)first * a.kv_heads + h;
        const int8_t* veb = a.v_exp + (long)first * a.kv_heads + h;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
          for (int i = 0; i < KL; ++i) __builtin_memcpy(&kr[kt][i], kb + (kt * 16 * row_bytes + k_off + i * 4 * CB), CB);
          if constexpr (E4M3) ke[kt] = keb[(unsigned)(kt * 16 + l16) * a.kv_heads];
        }
#pragma unroll
        for (int i = 0; i < VR; ++i) {
          load_v(vr[i], vb + ((F32 ? i : i * 64 / CPR) * row_bytes + v_off));
          if constexpr (E4M3) ve[i] = veb[(unsigned)v_key(i) * a.kv_heads];
        }
      } else {
        load_page(n0 + NW * BK);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const long r = __shfl(first, kt * 16 + l16);
          const char* src = static_cast<const char*>(a.k) + r * row_bytes + h * (DH * ES) + grp * CB;
#pragma unroll
          for (int i = 0; i < KL; ++i) __builtin_memcpy(&kr[kt][i], src + i * 4 * CB, CB);
          if constexpr (E4M3) ke[kt] = a.k_exp[r * a.kv_heads + h];
        }
#pragma unroll
        for (int i = 0; i < VR; ++i) {
          const long r = __shfl(first, v_key(i));
          const unsigned c = F32 ? l16 * VB : lane % CPR * CB;
          load_v(vr[i], static_cast<const char*>(a.v) + r * row_bytes + h * (DH * ES) + c);
          if constexpr (E4M3) ve[i] = a.v_exp[r * a.kv_heads + h];
        }
      }
    };
    load_page(key0 + wave * BK);

    // this lane's query head (heads past the group repeat its last one and are not stored);
    // the channels of slot grp at K load i are (i*4 + grp) * CE ..
    const long q_at = s * a.q_stride + (long)(h * a.group + min(g0 + l16, a.group - 1)) * DH;
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
    load(key0 + wave * BK);

    f32x4 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){};
    float m_run = -INFINITY, l_run = 0.f;
    for (int n0 = key0 + wave * BK; n0 < key1; n0 += NW * BK) {
      const unsigned keys = mask;
      const bool cut = keys != kAll;
      f32x4 sc[KT] = {};
      float vf[F32 ? 4 : 1][DT];
      if constexpr (F32) {
        // codes times their exponent before the products, which could overflow without it
        const float sk = E4M3 ? pow2(ke[0]) : 1.f;
#pragma unroll
        for (int i = 0; i < KL; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x[CE / 4];
            if constexpr (E4M3) {
              const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[0][i][j], false);
              const f32x2 up = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[0][i][j], true);
              x[0] = lo[0] * sk, x[1] = lo[1] * sk, x[2] = up[0] * sk, x[3] = up[1] * sk;
            } else {
              x[0] = __uint_as_float(kr[0][i][j]);
            }
#pragma unroll
            for (int u = 0; u < CE / 4; ++u) sc[0] = Mfma<16>::mul(x[u], qs[i * CE + j * (CE / 4) + u], sc[0]);
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
          // 0 * infinity: what a row that is not there holds must not enter the products
          if (cut && !(keys >> v_key(i) & 1))
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[i][dt] = 0.f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < VR; ++i) {
          const int f = i * 64 + lane, r = f / CPR;
          u32x4 x;
          __builtin_memcpy(&x, &vr[i], CB);
          const bool gone = cut && !(keys >> r & 1);
          if (gone) x = (u32x4){};  // 0 * infinity, as above
          if constexpr (E4M3) {
            // an exponent that was never written may be -128, as a scale a NaN that makes one of 0 too
            const float sv = pow2(gone ? 0 : ve[i]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              *reinterpret_cast<bf16x8*>(vl + r * DH + ((((f % CPR) * 2 + j) ^ swz(r)) * 8)) = widen(x[2 * j], x[2 * j + 1], sv);
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
              for (int j = 0; j < 2; ++j)
                sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(kr[kt][i][2 * j], kr[kt][i][2 * j + 1], sk),
                                                                 qb[i * 2 + j], sc[kt], 0, 0, 0);
            } else {
              sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[kt][i]), qb[i], sc[kt], 0, 0, 0);
            }
          }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // the V rows are in LDS
      }
      load(n0 + NW * BK);

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
        const float alpha = m_run == -INFINITY ? 0.f : rescale<F32>(m_run, m_new, a.scale);
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
      sh.m_part[wave][l16] = m_run;
      sh.l_part[wave][l16] = l_tot;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sh.buf[wave][l16 * P + (grp * 4 + e) * DT + dt] = acc[dt][e];
      } else {
        *reinterpret_cast<f32x4*>(&sh.buf[wave][l16 * P + dt * 16 + grp * 4]) = acc[dt];
      }
    }
    __syncthreads();
    const int n_heads = min(kRows, a.group - g0);
    for (int f = threadIdx.x; f < n_heads * (DH / 4); f += NW * kWave) {
      const int r = f / (DH / 4), c = (f - r * (DH / 4)) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int x = 0; x < NW; ++x) m = fmaxf(m, sh.m_part[x][r]);
      f32x4 sum = {};
      float l = 0.f;
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        const float mw = sh.m_part[x][r], lw = sh.l_part[x][r];
        if (mw == -INFINITY && lw == 0.f) continue;  // no key, or no finite score
        const float wt = rescale<F32>(mw, m, a.scale);
        l = fmaf(wt, lw, l);
        sum += wt * *reinterpret_cast<const f32x4*>(&sh.buf[x][r * P + c]);
      }
      if (!part) {
        write_out<F32, DH>(a, (long)s * (a.kv_heads * a.group) + h * a.group + g0 + r, c, m, l, sum);
      } else {
        *reinterpret_cast<f32x4*>(&part->o[r * DH + c]) = sum;
        if (c == 0) *reinterpret_cast<f32x2*>(&part->ml[2 * r]) = (f32x2){m, l};
      }
    }
  }
};

// one item per workgroup
template <bool F32, bool E4M3, int DH, bool ALIGNED>
__global__ __launch_bounds__(kWholeWaves * 64) void paged_whole_kernel(PagedArgs a, Plan plan) {
  typedef Attend<F32, E4M3, DH, ALIGNED, kWholeWaves> A;
  __shared__ __attribute__((aligned(16))) typename A::Shared sh;
  const int per = a.kv_heads * plan.gts;
  const int s = blockIdx.x / per, item = blockIdx.x - s * per, h = item / plan.gts;
  A::run(a, plan, sh, s, h, (item - h * plan.gts) * kRows, 0, uniform(seq_len(a, s)), nullptr);
}

// One run of tiles per workgroup. Two waves to a SIMD, stated: without it the
// compiler spreads the 128-wide forms over more registers than that leaves (48
// sequences of 201 to 8009 rows in bf16 94 -> 85 us).
template <bool F32, bool E4M3, int DH, bool ALIGNED>
__global__ __launch_bounds__(kSplitWaves * 64, 2) void paged_split_kernel(PagedArgs a, Plan plan) {
  typedef Attend<F32, E4M3, DH, ALIGNED, kSplitWaves> A;
  __shared__ __attribute__((aligned(16))) typename A::Shared sh;
  const int per = a.kv_heads * plan.gts;
  Walk walk;
  walk.view(a, per, 0, 0);
  const long total = all_tiles(a, per, walk), run = run_tiles(total, plan.wgs);
  const long begin = run * blockIdx.x, end = min(total, begin + run);
  Note note{0, 0, 0, 0};
  for (long pos = begin; pos < end;) {
    const int l = walk.find(a, per, pos);
    if (l < 0) break;  // lengths that changed under the call
    const int s = uniform(walk.s0 + l), len = __builtin_amdgcn_readlane(walk.len, l), tiles = tiles_of(len);
    const long off = pos - __shfl(walk.from, l);
    const int item = uniform((int)div_pos(off, tiles));
    const int t0 = uniform((int)(off - (long)item * tiles));
    const int n_t = uniform((int)min((long)(tiles - t0), end - pos));
    const int h = item / plan.gts;
    const int slot = pos == begin ? 0 : 1;
    Part<DH>* part = n_t == tiles ? nullptr : static_cast<Part<DH>*>(a.ws) + 2 * (long)blockIdx.x + slot;
    if (t0 == 0 && n_t < tiles)  // the run ends here
      note = Note{s, item, slot, (int)min(div_pos(pos + tiles - 1, run), (long)plan.wgs - 1) - (int)blockIdx.x};
    A::run(a, plan, sh, s, h, (item - h * plan.gts) * kRows, t0 * kTile, min(len, (t0 + n_t) * kTile), part);
    pos += n_t;
    if (pos < end) __syncthreads();  // the merge has read what the next item writes
  }
  if (threadIdx.x == 0) notes<DH>(a, plan)[blockIdx.x] = note;
}

template <bool F32, bool E4M3, int DH, bool ALIGNED>
hipError_t launch(const PagedArgs& a, hipStream_t s) {
  const long max_len = (long)a.max_pages * a.page_size;
  Plan plan{0, gts_of(a.group), FastDiv((uint32_t)a.page_size), 0, 1};
  if (!splits(a.n_seqs, a.kv_heads, a.group, max_len)) {
    hipLaunchKernelGGL((paged_whole_kernel<F32, E4M3, DH, ALIGNED>), dim3((unsigned)(a.n_seqs * a.kv_heads * plan.gts)),
                       dim3(kWholeWaves * 64), 0, s, a, plan);
    return hipGetLastError();
  }
  plan.wgs = workgroups(a.n_seqs, a.kv_heads, a.group, max_len);
  hipLaunchKernelGGL((paged_split_kernel<F32, E4M3, DH, ALIGNED>), dim3(plan.wgs), dim3(kSplitWaves * 64), 0, s, a, plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_join<F32, DH>(a, plan, s);
}

template <bool F32, int DH>
hipError_t launch_held(const PagedArgs& a, bool e4m3, hipStream_t s) {
  // a block of 32 rows lies in one page where the page size is a multiple of 32
  if (a.page_size % 32 == 0) return e4m3 ? launch<F32, true, DH, true>(a, s) : launch<F32, false, DH, true>(a, s);
  return e4m3 ? launch<F32, true, DH, false>(a, s) : launch<F32, false, DH, false>(a, s);
}

}  // namespace

// Asked for as if every item were dealt from kLeastWhole rows on, so that a workspace
// made for n_seqs and max_len serves fewer sequences too; over e2m1 rows as if items were taken four abreast.
size_t paged_attention_bytes(int n_seqs, int kv_heads, int group, int head_dim, long max_len, bool e2m1) {
  if (n_seqs <= 0 || max_len <= kLeastWhole) return 0;
  const long tiles = (long)n_seqs * kv_heads * gts_of(group) * ((max_len + kTile - 1) / kTile);
  const long runs = e2m1 ? std::min((long)kMostRuns, tiles) : workgroups(n_seqs, kv_heads, group, max_len);
  return (size_t)runs * (2 * kRows * (head_dim + 2) * sizeof(float) + sizeof(Note));
}

hipError_t launch_paged_attention(const PagedArgs& a, bool bf16, Held held, int head_dim, hipStream_t s) {
  if (a.n_seqs <= 0) return hipSuccess;
  if (held == kE2M1) return launch_paged_attention_e2m1(a, bf16, head_dim, s);
  const bool e4m3 = held == kE4M3;
  if (bf16) return head_dim == 64 ? launch_held<false, 64>(a, e4m3, s) : launch_held<false, 128>(a, e4m3, s);
  return head_dim == 64 ? launch_held<true, 64>(a, e4m3, s) : launch_held<true, 128>(a, e4m3, s);
}

}  // namespace hsa
