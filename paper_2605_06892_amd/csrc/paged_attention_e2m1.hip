// Attention of one query per sequence over pages of e2m1 rows: 17/32 of a byte for each value. Items, parts and joins are those
// of the other caches (paged.h). What bounds it is how the memory is read.
//
// A head's row is 64 bytes of 128 channels, half a line of the caches, so the items of a sequence are read together:
// up to four neighbouring ones by the waves of one workgroup, and all of them, over the same rows, by workgroups that
// follow each other on one XCD, whose L2 then has each line once. Each item's tiles are dealt out in runs that are cut at
// the same tiles for all. Four sequences of 30011 to 131072 rows, 8 heads of 128: in the other caches' order 735 MB are
// fetched for 316 and it takes 123 us; with the order alone 321 MB and 96 us, of which loading takes 82 (that alone, with
// four items abreast, 72).
//
// A block of 32 keys is five loads (two of K, two of V, one of exponents, V's in the lower lanes and K's in the
// upper), one block ahead: 48 sequences of 201 to 8009 rows in pages of 16 57 us with 20 loads to a block, of single exponents
// and of 4 bytes of V by each lane, 37 so. Two blocks ahead took longer, 75 -> 81 for the four sequences (it is not
// the latency that bounds it). K goes from its loads to the products: slot lane / 16 has a quarter of a
// head's channels, which share an exponent, the operand of the conversion to bf16. V's codes and all exponents go
// through LDS, where a lane reads DT neighbouring channels of its slot's 8 keys and pairs keys in registers, as the
// products contract over them. Nothing but the probabilities is rounded to bf16, as in the other forms.
//
// fp32 queries are three bf16 parts, cut from the top, and so are the probabilities: three products in the place of one
// are exact to fp32's 24 bits (less what lies under 2^-133, bf16's least), and take a fifth of the time of the fp32
// matrix instructions: the same sequences 215 us with those, 97 so; bf16 queries 75.
#include "paged.h"

#include <type_traits>

namespace hsa {
namespace {

constexpr int kWaves = 8;

// The loads of a block do not depend on whether there is such a block: where there is none they read the cache's first
// row, so that a wait for one block leaves the later one under way.
template <bool F32, int DH, bool ALIGNED>
struct Attend {
  static constexpr int NW = kWaves, PARTS = F32 ? 3 : 1;  // waves; bf16 parts of a query and of a probability
  static constexpr int BK = 32, KT = 2, DT = DH / 16;
  static constexpr int P = DH + 4;                     // padded row of the merge buffer, floats
  static constexpr int HB = DH / 2, HX = DH / kGroup;  // bytes of a head's row, its exponents
  static constexpr int KB = HB / 4;                    // of K per lane and key tile
  static constexpr int VR = BK * HB / 1024, VPR = HB / 16;  // V loads of a lane, of a row
  // V in LDS: 4 rows together and a row's bytes between them, so that the reads of 4 slots' rows fall into different banks
  static constexpr int VS = 5 * HB, VX = BK / 4 * VS;  // bytes of 4 rows; where the exponents are, a word for each row of V, then of K
  struct Shared {
    float buf[NW][kRows * P];  // V rows, then the merge
    float m_part[NW][kRows], l_part[NW][kRows];
  };
  static_assert(VX + 2 * BK * 4 <= kRows * P * 4, "a block's codes and exponents fit");
  struct Block {
    unsigned k[KT][KB / 4];
    u32x4 v[VR];
    unsigned x;      // exponents of V's row `lane`, of K's row lane - 32
    unsigned mask;   // keys that there are
  };

  // Keys key0 .. key1-1 for plan.abreast items from `item` on, all uniform: wave w takes item + w % abreast and every
  // (NW / abreast)-th block. part: where the first one's unnormalized result goes, the others' `stride` parts on; NULL
  // for the outputs themselves.
  static __device__ __forceinline__ void run(const PagedArgs& a, const Plan& plan, Shared& sh, int s, int item,
                                             int key0, int key1, Part<DH>* part, long stride) {
    const int lane = threadIdx.x & 63;
    const int wave = uniform(threadIdx.x >> 6), abreast = plan.abreast;
    const int l16 = lane & 15, grp = lane >> 4;
    const int sub = wave & (abreast - 1), turns = NW / abreast;
    const int h = (item + sub) / plan.gts, g0 = (item + sub - h * plan.gts) * kRows;
    const unsigned row_bytes = (unsigned)a.kv_heads * HB, row_exps = (unsigned)a.kv_heads * HX;
    const float sl2e = a.scale * kLog2e;
    const int32_t* pages = a.page_table + (long)s * a.max_pages;
    char* vl = reinterpret_cast<char*>(sh.buf[wave]);
    const char* kc = static_cast<const char*>(a.k) + h * HB;
    const char* vc = static_cast<const char*>(a.v) + h * HB;
    const int8_t* xc = (lane < BK ? a.v_exp : a.k_exp) + h * HX;

    // Pages. ALIGNED: a block lies in one; lane i holds the number of page `base` + i of the sequence, for 64
    // pages at a time. Else: this lane's key's, of the block after the one loaded last.
    int page, base = -kWave;
    auto load_page = [&](int n0) { page = pages[plan.page.quot(min(n0 + lane % BK, key1 - 1))]; };
    auto load = [&](Block& b, int n0) {
      int first;
      if constexpr (ALIGNED) {
        const int n = min(n0, key1 - 1), at = uniform((int)plan.page.quot(n));
        if (at >= base + kWave) {
          base = at;
          page = pages[min(base + lane, (int)plan.page.quot(key1 - 1))];
          asm volatile("" : "+v"(page));  // waited for here, not where the blocks' loads are under way
        }
        const int number = __builtin_amdgcn_readlane(page, at - base);
        const bool ok = n0 < key1 && number >= 0 && number < a.n_pages;
        first = ok ? number * a.page_size + (n0 - at * a.page_size) : 0;
        b.mask = !ok ? 0u : key1 - n0 >= BK ? ~0u : (1u << (key1 - n0)) - 1;
      } else {
        const int t = n0 + lane % BK;
        const bool ok = t < key1 && page >= 0 && page < a.n_pages;
        first = ok ? page * a.page_size + (t - (int)plan.page.quot(t) * a.page_size) : 0;
        b.mask = (unsigned)__ballot(ok);
        load_page(n0 + turns * BK);
      }
      auto row = [&](int r) { return (long)(ALIGNED ? first + r : __shfl(first, r)); };
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) __builtin_memcpy(b.k[kt], kc + row(kt * 16 + l16) * row_bytes + grp * KB, KB);
#pragma unroll
      for (int i = 0; i < VR; ++i) {
        const int f = i * 64 + lane;
        b.v[i] = *reinterpret_cast<const u32x4*>(vc + row(f / VPR) * row_bytes + f % VPR * 16);
      }
      b.x = 0;
      __builtin_memcpy(&b.x, xc + (ALIGNED ? first + lane % BK : first) * (long)row_exps, HX);
    };

    // this lane's query head (heads past the group repeat its last one and are not stored): slot grp has a quarter of the channels
    const long q_at = s * a.q_stride + (long)(h * a.group + min(g0 + l16, a.group - 1)) * DH + grp * (DH / 4);
    bf16x8 qb[DH / 32][PARTS];
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) {
      if constexpr (F32) {
        const float* q = static_cast<const float*>(a.q) + q_at + i * 8;
        const f32x4u x[2] = {*reinterpret_cast<const f32x4u*>(q), *reinterpret_cast<const f32x4u*>(q + 4)};
        const float y[8] = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
        cut3(y, qb[i]);
      } else {
        qb[i][0] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.q) + q_at + i * 8);
      }
    }

    f32x4 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = (f32x4){};
    float m_run = -INFINITY, l_run = 0.f;
    auto attend = [&](Block& b, int n_next) {
      const unsigned keys = b.mask;
      const bool cut = keys != ~0u;
#pragma unroll
      for (int i = 0; i < VR; ++i) {  // neither codes nor exponents of rows that are not there (-128 makes a NaN of 0 too)
        const int f = i * 64 + lane, r = f / VPR;
        if (cut && !(keys >> r & 1)) b.v[i] = (u32x4){};
        *reinterpret_cast<u32x4*>(vl + r / 4 * VS + r % 4 * HB + f % VPR * 16) = b.v[i];
      }
      if (cut && lane < BK && !(keys >> lane & 1)) b.x = 0;
      *reinterpret_cast<unsigned*>(vl + VX + lane * 4) = b.x;
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      f32x4 sc[KT] = {};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const float sk = pow2(*reinterpret_cast<const int8_t*>(vl + VX + (BK + kt * 16 + l16) * 4 + grp * (DH / 4) / kGroup));
#pragma unroll
        for (int j = 0; j < KB / 4; ++j) {
          const bf16x8 y = widen4(b.k[kt][j], sk);
#pragma unroll
          for (int x = PARTS - 1; x >= 0; --x) sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, qb[j][x], sc[kt], 0, 0, 0);
        }
      }
      load(b, n_next);

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
      bf16x8 pf[PARTS];
      if constexpr (F32) {
        const float y[8] = {sc[0][0], sc[0][1], sc[0][2], sc[0][3], sc[1][0], sc[1][1], sc[1][2], sc[1][3]};
        cut3(y, pf);
      } else {
        pf[0] = __builtin_shufflevector(to_bf16x4(sc[0]), to_bf16x4(sc[1]), 0, 1, 2, 3, 4, 5, 6, 7);
      }
      // this lane's DT channels of its slot's 8 keys, as the probabilities have them
      const u32x4 e0 = *reinterpret_cast<const u32x4*>(vl + VX + grp * 16), e1 = *reinterpret_cast<const u32x4*>(vl + VX + 64 + grp * 16);
      bf16x2 v2[DT / 2][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        unsigned c = 0;
        __builtin_memcpy(&c, __builtin_assume_aligned(vl + (grp + (i >> 2) * 4) * VS + (i & 3) * HB + l16 * (DT / 2), DT / 2), DT / 2);
        const float sv = pow2((int8_t)((i < 4 ? e0[i] : e1[i & 3]) >> (8 * (l16 * DT / kGroup))));
        v2[0][i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, sv, 0);
        v2[1][i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, sv, 1);
        if constexpr (DT == 8) {
          v2[2][i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, sv, 2);
          v2[3][i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, sv, 3);
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        bf16x8 vf;
#pragma unroll
        for (int i = 0; i < 8; ++i) vf[i] = v2[dt / 2][i][dt & 1];
#pragma unroll
        for (int x = PARTS - 1; x >= 0; --x) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[x], acc[dt], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // read before the next block's rows
    };
    int n0 = key0 + wave / abreast * BK;
    if (n0 < key1) {
      Block b;
      if constexpr (!ALIGNED) load_page(n0);
      load(b, n0);
      for (; n0 < key1; n0 += turns * BK) attend(b, n0 + turns * BK);
    }

    // merge of the waves. acc[dt][e] is channel (grp*4 + e)*DT + dt of row l16
    float l_tot = l_run + __shfl_xor(l_run, 16);
    l_tot += __shfl_xor(l_tot, 32);
    if (grp == 0) {
      sh.m_part[wave][l16] = m_run;
      sh.l_part[wave][l16] = l_tot;
    }
#pragma unroll
    for (int dt = 0; dt < DT; dt += 4)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(&sh.buf[wave][l16 * P + (grp * 4 + e) * DT + dt]) =
            (f32x4){acc[dt][e], acc[dt + 1][e], acc[dt + 2][e], acc[dt + 3][e]};
    __syncthreads();
    auto join = [&](auto abreast_c) {
      constexpr int A = decltype(abreast_c)::value;
      const int rows = min(kRows, a.group);
      for (int f = threadIdx.x; f < A * rows * (DH / 4); f += NW * kWave) {
        const int of = f / (DH / 4), x0 = of / rows, r = of - x0 * rows, c = (f - of * (DH / 4)) * 4;
        const int hh = (item + x0) / plan.gts, g = (item + x0 - hh * plan.gts) * kRows + r;
        if (g >= a.group) continue;
        float m = -INFINITY;
#pragma unroll
        for (int x = 0; x < NW; x += A) m = fmaxf(m, sh.m_part[x0 + x][r]);
        f32x4 sum = {};
        float l = 0.f;
#pragma unroll
        for (int x = 0; x < NW; x += A) {
          const float mw = sh.m_part[x0 + x][r], lw = sh.l_part[x0 + x][r];
          if (mw == -INFINITY && lw == 0.f) continue;  // no key, or no finite score
          const float wt = rescale<F32>(mw, m, a.scale);
          l = fmaf(wt, lw, l);
          sum += wt * *reinterpret_cast<const f32x4*>(&sh.buf[x0 + x][r * P + c]);
        }
        if (!part) {
          write_out<F32, DH>(a, (long)s * (a.kv_heads * a.group) + hh * a.group + g, c, m, l, sum);
        } else {
          Part<DH>* to = part + x0 * stride;
          *reinterpret_cast<f32x4*>(&to->o[r * DH + c]) = sum;
          if (c == 0) *reinterpret_cast<f32x2*>(&to->ml[2 * r]) = (f32x2){m, l};
        }
      }
    };
    if (abreast == 1) join(std::integral_constant<int, 1>{});
    else if (abreast == 2) join(std::integral_constant<int, 2>{});
    else join(std::integral_constant<int, 4>{});
  }
};

// one item, or a few abreast, per workgroup
template <bool F32, int DH, bool ALIGNED>
__global__ __launch_bounds__(kWaves * 64, 2) void e2m1_whole_kernel(PagedArgs a, Plan plan) {
  typedef Attend<F32, DH, ALIGNED> A;
  __shared__ __attribute__((aligned(16))) typename A::Shared sh;
  const int per = a.kv_heads * plan.gts / plan.abreast;
  const int b = xcd_contiguous(blockIdx.x, gridDim.x), s = b / per;
  A::run(a, plan, sh, s, (b - s * per) * plan.abreast, 0, uniform(seq_len(a, s)), nullptr, 0);
}

// Run `rank` of items item .. item + abreast-1 per workgroup, its parts and notes those of runs (item + x) *
// plan.runs + rank. Without plan.runs (more items than runs) one run of all items' tiles.
template <bool F32, int DH, bool ALIGNED>
__global__ __launch_bounds__(kWaves * 64, 2) void e2m1_split_kernel(PagedArgs a, Plan plan) {
  typedef Attend<F32, DH, ALIGNED> A;
  __shared__ __attribute__((aligned(16))) typename A::Shared sh;
  const int items = a.kv_heads * plan.gts;
  int rank = blockIdx.x, own = -1, per = items;
  long id = blockIdx.x;
  if (plan.runs > 0) {
    const int beside = items / plan.abreast, slot = blockIdx.x / kXcds;
    rank = slot / beside * kXcds + blockIdx.x % kXcds;
    own = (slot - slot / beside * beside) * plan.abreast;
    id = (long)own * plan.runs + rank;
    per = 1;
  }
  const int runs = plan.runs > 0 ? plan.runs : plan.wgs;
  Walk walk;
  walk.view(a, per, 0, 0);
  const long total = all_tiles(a, per, walk), run = run_tiles(total, runs);
  const long begin = run * rank, end = min(total, begin + run);
  Note note{0, 0, 0, 0};
  for (long pos = begin; pos < end;) {
    const int l = walk.find(a, per, pos);
    if (l < 0) break;  // lengths that changed under the call
    const int s = uniform(walk.s0 + l), len = __builtin_amdgcn_readlane(walk.len, l), tiles = tiles_of(len);
    const long off = pos - __shfl(walk.from, l);
    const int nth = uniform((int)div_pos(off, tiles)), item = own < 0 ? nth : own;
    const int t0 = uniform((int)(off - (long)nth * tiles));
    const int n_t = uniform((int)min((long)(tiles - t0), end - pos));
    const int slot = pos == begin ? 0 : 1;
    Part<DH>* part = n_t == tiles ? nullptr : static_cast<Part<DH>*>(a.ws) + 2 * id + slot;
    if (t0 == 0 && n_t < tiles)  // the run ends here
      note = Note{s, item, slot, (int)min(div_pos(pos + tiles - 1, run), (long)runs - 1) - rank};
    A::run(a, plan, sh, s, item, t0 * kTile, min(len, (t0 + n_t) * kTile), part, 2L * plan.runs);
    pos += n_t;
    if (pos < end) __syncthreads();  // the merge has read what the next item writes
  }
  if ((int)threadIdx.x < plan.abreast) {
    note.item += threadIdx.x;
    notes<DH>(a, plan)[id + (long)threadIdx.x * plan.runs] = note;
  }
}

// How many items a workgroup takes at once, and the runs of each.
struct Shape {
  int abreast, runs, wgs;  // wgs: runs of all items
};
Shape shape(int n_seqs, int kv_heads, int group, long max_len) {
  const long items = (long)kv_heads * gts_of(group), cus = compute_units();
  const long tiles = (long)n_seqs * ((max_len + kTile - 1) / kTile);  // of an item
  int abreast = items % 4 == 0 ? 4 : items % 2 == 0 ? 2 : 1;
  while (abreast > 1 && tiles * items < 2 * cus * abreast) abreast >>= 1;  // too few to go round
  const long runs = std::min(std::min(cus * abreast, (long)kMostRuns) / items, tiles) / kXcds * kXcds;
  if (runs > 0) return {abreast, (int)runs, (int)(runs * items)};
  return {1, 0, workgroups(n_seqs, kv_heads, group, max_len)};
}

template <bool F32, int DH, bool ALIGNED>
hipError_t launch(const PagedArgs& a, hipStream_t s) {
  const long max_len = (long)a.max_pages * a.page_size, items = (long)a.kv_heads * gts_of(a.group);
  Plan plan{0, gts_of(a.group), FastDiv((uint32_t)a.page_size), 0, 1};
  if (!splits(a.n_seqs, a.kv_heads, a.group, max_len)) {
    // abreast where that leaves a workgroup for each CU (64 sequences of 100 to 700 rows, 8 heads: 17.7 us one by one, 14.4 four abreast)
    if (items * a.n_seqs >= 4 * compute_units()) plan.abreast = items % 4 == 0 ? 4 : items % 2 == 0 ? 2 : 1;
    hipLaunchKernelGGL((e2m1_whole_kernel<F32, DH, ALIGNED>), dim3((unsigned)(a.n_seqs * items / plan.abreast)), dim3(kWaves * 64), 0, s, a, plan);
    return hipGetLastError();
  }
  const Shape p = shape(a.n_seqs, a.kv_heads, a.group, max_len);
  plan.wgs = p.wgs;
  plan.runs = p.runs;
  plan.abreast = p.abreast;
  hipLaunchKernelGGL((e2m1_split_kernel<F32, DH, ALIGNED>), dim3(p.wgs / p.abreast), dim3(kWaves * 64), 0, s, a, plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_join<F32, DH>(a, plan, s);
}

template <bool F32, int DH>
hipError_t launch_aligned(const PagedArgs& a, hipStream_t s) {
  // a block of 32 rows lies in one page where the page size is a multiple of 32
  return a.page_size % 32 == 0 ? launch<F32, DH, true>(a, s) : launch<F32, DH, false>(a, s);
}

}  // namespace

hipError_t launch_paged_attention_e2m1(const PagedArgs& a, bool bf16, int head_dim, hipStream_t s) {
  if (bf16) return head_dim == 64 ? launch_aligned<false, 64>(a, s) : launch_aligned<false, 128>(a, s);
  return head_dim == 64 ? launch_aligned<true, 64>(a, s) : launch_aligned<true, 128>(a, s);
}

}  // namespace hsa
