// Rows times weights in e2m1 groups: y = act(s (x W^T)) + r for a few rows, bound by reading W.
//
// A wave takes 16 outputs (the rows of the matrix instructions' tile) and units of 512 inputs. In each of
// a unit's four steps a lane loads 16 bytes, the 32 codes of one group, 64 bytes of one row for its four
// lanes; the exponents of all four are one load before them (a byte of its own for every step, of 16 rows each, took a
// quarter of the time). The conversion to bf16 takes the exponent as its operand: exact, one
// instruction for two weights, and no scaling of sums. Slot lane / 16 of the contraction holds that group, 8 values to an
// instruction; x is read from LDS in the same order. The rows of x are the tile's columns.
// Codes are loaded a unit ahead of the products, each step's into the registers that its products have
// freed; the waves of a workgroup that share inputs (`outs` of them) load x together, those that share
// outputs (`splits`) take units in turn and are joined in LDS.
//
// fp32 rows are taken as three bf16 parts, cut from the top: 8 + 8 + 8 bits are all that fp32 has, so every
// product is exact here too, and sums are in fp32 as before (what of a value lies under 2^-133, bf16's least, is
// left out). The parts are columns of their own, five rows to a tile, summed at the end. The fp32
// matrix instructions are 16 times slower than the bf16 ones: 5 rows of 8960 by 1537 outputs take 16 us with them,
// 9.7 so, of 8192 by 16384 48 and 21.
//
// One row of 8192 by 32768 outputs: 30 us, 4.7 TB/s; 16 rows 37 us.
#include "seq_common.h"

#include <algorithm>
#include <type_traits>

namespace hsa {
namespace {

constexpr int kOuts = 16;   // outputs of a tile, and columns for rows of x
constexpr int kUnit = 512;  // inputs of a unit: 16 groups, four steps
constexpr int kUnitGroups = kUnit / kGroup;
constexpr int kMostWaves = 8;

__device__ __forceinline__ float gelu_exact(float x) {
  const float y = 0.7978845608028654f * fmaf(0.044715f * x, x * x, x);
  return x / (1.f + expf(-2.f * y));
}

// Workgroups of splits * outs waves; NT tiles of rows of x; XS rows of x loaded by each wave of a split.
template <bool BF16, int NT, int XS>
__global__ __launch_bounds__(kMostWaves * kWave) void linear_w4_kernel(LinearW4 a, int outs, int splits) {
  constexpr int PARTS = BF16 ? 1 : 3;           // rows in LDS of a row of x
  constexpr int ROWS = NT * (BF16 ? kOuts : 5); // rows of x of a workgroup
  constexpr int XL = BF16 ? 1 : 2;              // loads of 16 bytes for 8 values
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int ks = wave / outs, no = wave - ks * outs;
  const int l16 = lane & 15, grp = lane >> 4;
  const int o0 = blockIdx.x * (kOuts * outs), m0 = blockIdx.y * ROWS;
  const int rows = min(a.rows - m0, ROWS), x_rows = XS * outs * PARTS;
  const int groups = a.d_in / kGroup, units = (groups + kUnitGroups - 1) / kUnitGroups;
  // outputs past the last repeat it and are not stored
  const long w_row = min(o0 + no * kOuts + l16, a.d_out - 1);
  const uint8_t* w = a.w + w_row * (a.d_in / 2);
  const int8_t* exps = a.exps + w_row * groups;

  // x of a unit in LDS, two units of each split (one where a wave reads what it wrote itself): row r at r * 1 KB, its
  // 16-byte chunk c at c ^ (r & 7), so that 8 rows' reads of one chunk spread over the banks. Rows past the last repeat it.
  const int bufs = outs > 1 ? 2 : 1;
  char* xl = lds + ks * bufs * x_rows * 1024;
  u32x4 xr[XS][XL];
  auto load_x = [&](int u) {
    const int k = min(u * kUnit + lane * 8, a.d_in - 8);
#pragma unroll
    for (int i = 0; i < XS; ++i) {
      const char* p = static_cast<const char*>(a.x) + ((long)(m0 + min(i * outs + no, rows - 1)) * a.d_in + k) * (BF16 ? 2 : 4);
#pragma unroll
      for (int j = 0; j < XL; ++j) xr[i][j] = *reinterpret_cast<const u32x4*>(p + j * 16);
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < XS; ++i) {
      bf16x8 part[PARTS];
      if constexpr (BF16) {
        part[0] = __builtin_bit_cast(bf16x8, xr[i][0]);
      } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(xr[i][j >> 2][j & 3]);
        cut3(x, part);
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const int r = (i * outs + no) * PARTS + p;
        *reinterpret_cast<bf16x8*>(xl + (buf * x_rows + r) * 1024 + (lane ^ (r & 7)) * 16) = part[p];
      }
    }
  };
  int x_row[NT];  // of this lane's column
#pragma unroll
  for (int t = 0; t < NT; ++t) x_row[t] = min(t * (BF16 ? kOuts : 15) + l16, rows * PARTS - 1);

  u32x4 c[4], e, e_next;  // codes of the steps; exponents, a word for each step
  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = (f32x4){};
  auto load_c = [&](int u, int i) {  // of a whole unit
    c[i] = *reinterpret_cast<const u32x4*>(w + (long)(u * kUnitGroups + i * 4 + grp) * 16);
  };
  auto multiply = [&](int i, int buf, bool gone) {
    bf16x8 x[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[t][j] = *reinterpret_cast<const bf16x8*>(xl + (buf * x_rows + x_row[t]) * 1024 + ((i * 16 + grp * 4 + j) ^ (x_row[t] & 7)) * 16);
        if (gone) x[t][j] = (bf16x8){};
      }
    const float s = pow2((int8_t)(e[i] >> (8 * grp)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x8 y = widen4(c[i][j], s);
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x[t][j], acc[t], 0, 0, 0);
    }
  };
  auto meet = [&] {
    if (outs > 1) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  };
  // whole units, as many in every split
  const int turns = a.d_in / kUnit / splits;
  int buf = 0;
  auto unit = [&](int u, auto more) {
    meet();  // this unit's x is in LDS, and the last one's has been read
    if constexpr (more) {
      __builtin_memcpy(&e_next, exps + (u + splits) * kUnitGroups, 16);
      load_x(u + splits);
      __builtin_amdgcn_sched_barrier(0);  // loads stay where they are
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      multiply(i, buf, false);
      if constexpr (more) {
        load_c(u + splits, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    buf ^= bufs - 1;
    if constexpr (more) {
      stage(buf);
      e = e_next;
    }
  };
  if (turns > 0) {
    int u = ks;
    load_x(u);
    __builtin_memcpy(&e, exps + u * kUnitGroups, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_c(u, i);
    stage(0);
    for (int t = 1; t < turns; ++t, u += splits) unit(u, std::true_type{});
    unit(u, std::false_type{});
  }
  // what is left: fewer units than splits, the last one perhaps of fewer groups
  if (turns * splits < units) {
    const int u = turns * splits + ks, at = min(u, units - 1);
    load_x(at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = min(at * kUnitGroups + i * 4 + grp, groups - 1);
      c[i] = *reinterpret_cast<const u32x4*>(w + (long)g * 16);
      e[i] = (unsigned)(uint8_t)exps[g] << (8 * grp);
    }
    stage(buf);
    meet();
#pragma unroll
    for (int i = 0; i < 4; ++i) multiply(i, buf, u * kUnitGroups + i * 4 + grp >= groups);  // inputs of 0 past the last
  }
  __syncthreads();

  // the splits' sums. acc[t][e]: output o0 + no * 16 + grp * 4 + e, column l16 of tile t
  f32x4* parts = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int t = 0; t < NT; ++t) parts[(wave * NT + t) * kWave + lane] = acc[t];
  __syncthreads();
  constexpr int PER = BF16 ? kOuts : 5;  // rows of a tile
  for (int f = threadIdx.x; f < outs * NT * 4 * PER; f += blockDim.x) {
    const int tile = f / (4 * PER), slot = f / PER % 4, r = f % PER;
    const int m = m0 + tile % NT * PER + r, o = o0 + tile / NT * kOuts + slot * 4;
    if (m >= a.rows) continue;
    f32x4 sum = {};
    for (int x = 0; x < splits; ++x)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) sum += parts[(x * outs * NT + tile) * kWave + slot * kOuts + r * PARTS + p];
    if (a.row_scale) sum *= a.row_scale[m];
    const long at = (long)m * a.d_out + o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.d_out) break;
      float z = sum[j];
      if constexpr (BF16) {
        if (a.gelu) z = gelu_tanh(z);
        if (a.residual) z += (float)static_cast<const bf16*>(a.residual)[at + j];
        if (a.out_f32) static_cast<float*>(a.y)[at + j] = z;
        else static_cast<bf16*>(a.y)[at + j] = (bf16)z;
      } else {
        if (a.gelu) z = gelu_exact(z);
        if (a.residual) z += static_cast<const float*>(a.residual)[at + j];
        static_cast<float*>(a.y)[at + j] = z;
      }
    }
  }
}

template <bool BF16, int NT, int XS>
hipError_t launch(const LinearW4& a, int outs, int splits, hipStream_t s) {
  constexpr int ROWS = NT * (BF16 ? kOuts : 5);
  const unsigned wgs = (unsigned)((a.d_out + outs * kOuts - 1) / (outs * kOuts)), tiles = (unsigned)((a.rows + ROWS - 1) / ROWS);
  const int lds = std::max(splits * (outs > 1 ? 2 : 1) * XS * outs * (BF16 ? 1 : 3), outs * splits * NT) * 1024;
  hipLaunchKernelGGL((linear_w4_kernel<BF16, NT, XS>), dim3(wgs, tiles), dim3(outs * splits * kWave), lds, s, a, outs, splits);
  return hipGetLastError();
}

template <int NT>
hipError_t launch_bf16(const LinearW4& a, int outs, int splits, hipStream_t s) {
  const int per = (std::min(a.rows, NT * kOuts) + outs - 1) / outs;  // rows of x for each wave
  // as many as a launch below may ask for
  if constexpr (NT == 1) {
    if (per <= 1) return launch<true, NT, 1>(a, outs, splits, s);
    if (per <= 2) return launch<true, NT, 2>(a, outs, splits, s);
    if (per > 8) return launch<true, NT, 16>(a, outs, splits, s);
  }
  if constexpr (NT < 4) {
    if (per <= 4) return launch<true, NT, 4>(a, outs, splits, s);
  }
  return launch<true, NT, 8>(a, outs, splits, s);
}

template <int NT>
hipError_t launch_f32(const LinearW4& a, int outs, int splits, hipStream_t s) {
  const int per = (std::min(a.rows, NT * 5) + outs - 1) / outs;
  // as many as a launch below may ask for
  if constexpr (NT < 4) {
    if (per <= 1) return launch<false, NT, 1>(a, outs, splits, s);
  }
  if (per <= 2) return launch<false, NT, 2>(a, outs, splits, s);
  if constexpr (NT == 1) {
    if (per > 3) return launch<false, NT, 5>(a, outs, splits, s);
  }
  return launch<false, NT, 3>(a, outs, splits, s);
}

}  // namespace

// Tiles of rows, waves that share inputs and waves that share outputs: as many of the former as leave half of the CUs a workgroup
// or more, for they share what is read of x (in one tile of bf16 rows 2 from one tile of outputs per CU on, 4 from two or two and a half
// on; few outputs and more than 16 rows take 2 all the same), and the latter where there is enough to split. The limits lie between
// the sizes below whose best shapes differ; where between them the shapes cross was not measured. Waves that share nothing else
// as many as up to 8 take the units in equally many turns, for what is left over is loaded without a turn before it. 5 fp32 rows,
// 10 units: 5 splits 7.0 us, 4 7.9, 6 7.6, 8 8.0; 16 units: 8 7.9, 4 8.6, 6 9.6; 18: 6 9.7, 4 10.8, 8 10.1; 27: 7 13.1, 4 14.3,
// 8 13.9; 4 bf16 rows, 7 units: 7 4.4, 4 5.0; 10: 5 5.1, 4 5.7; 18 and 32 within 2%. Waves x splits, us:
//                          1x4  2x2  4x1  4x2  8x1             2 tiles 4x1  8x1   4 tiles 8x1
//    4 rows, 8960 x 1536   6.6  8.5 12.7 12.6 22.5
//    4       5120 x 5120   9.2  7.4 10.9 10.3 18.2
//   16       1536 x 8960   9.8  6.6  5.3  6.7  6.9
//   16       8192 x 32768   64   39   38   38   37
//   32       5120 x 16384                  22   21                   18     25       28
//   32       8192 x 32768             63   63   58                   45     42       49
//   64       5120 x 16384             37   36   33                   27     24       35
//   64       8192 x 32768            112  112  102                   78     67       56
//                          2x2  4x1  4x2             2 tiles 4x2  4x1  8x1
//    1 row,  8192 x 8192   10.4 15.1 14.0
//   16       8192 x 8192   13.5 18.4 17.8
//   16       2048 x 8192    5.6  5.9
//   16       5120 x 10240  14.6 13.2 13.2                         13.8
//   32       5120 x 5120   12.1 12.6 12.1                    15.8 16.6 23.7
//   32       8192 x 8192   20.3 18.4 17.4                    21.9 23.6 33.4
//   32       5120 x 10240  17.9 17.0 18.0                    16.2 16.9
//   64       5120 x 5120   17.1 16.5 17.1                    15.7 16.6 22.9
//   64       8192 x 8192   33.7 29.0 28.9                    22.7 24.4 32.4
//   64       5120 x 10240  27.8 27.9 26.1                    27.3 23.3 23.4
// (4x2 of two tiles fill a CU's LDS: good where one turn of them fills the CUs.)
// fp32 rows: cutting them is most of the work, so as many waves share x as leave the CUs filled. us:
//                          1 tile 4x2  8x1        2 tiles 4x1  4x2  8x1   4 tiles 8x1
//    5 rows, 8192 x 32768      38.5   35.9
//    8       5120 x 5120       11.8   18.3              15.4  13.8 20.9        26.1
//    8       8192 x 16384      35.6   29.0              26.1  24.4 30.6        39.4
//   16       5120 x 5120       20.1   17.5              17.3  15.2 21.6        29.2
//   16       5120 x 13824      39.8   31.8              25.3  27.7 23.2        29.7
//   16       8192 x 16384      61.7   47.6              39.6  42.5 36.2        44.1
//   16       8192 x 32768       123   97.9              77.6  84.1 74.4        53.0
//   64       1536 x 8960       47.6   18.4              17.1  30.4 17.2        23.6
//   64       5120 x 5120       46.5   39.3              35.4  39.4 40.3        33.2
//   64       8192 x 16384       183    145               123   138  121         102
hipError_t launch_linear_w4(const LinearW4& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0 || a.d_out <= 0) return hipSuccess;
  const long outs = (a.d_out + kOuts - 1) / kOuts, cus = compute_units();
  const int units = (a.d_in + kUnit - 1) / kUnit;
  const bool some = outs >= cus;
  const int four = units >= 8 ? 2 : 1, two = units >= 2 ? 2 : 1, turns = (units + 7) / 8, one = (units + turns - 1) / turns;  // splits beside 4, 2 and 1
  if (!bf16) {
    auto groups = [&](int rows, int waves) { return (a.rows + rows - 1) / rows * ((outs + waves - 1) / waves); };
    auto full = [&](long n) { return (double)n / ((n + cus - 1) / cus * cus); };  // of the CUs, in as many turns as n need
    if (a.rows > 10 && full(groups(20, 8)) >= 0.75) return launch_f32<4>(a, 8, 1, s);
    if (a.rows > 5) {
      if (full(groups(10, 8)) >= 0.6) return launch_f32<2>(a, 8, 1, s);
      const long n = groups(10, 4);
      if (n >= 0.6 * cus) return launch_f32<2>(a, 4, n >= 2 * cus ? 1 : four, s);
    }
    if (outs >= 8 * cus) return launch_f32<1>(a, 8, 1, s);
    if (outs >= 2 * cus || (some && a.rows > 5)) return launch_f32<1>(a, 4, four, s);
    return some ? launch_f32<1>(a, 2, two, s) : launch_f32<1>(a, 1, one, s);
  }
  if (a.rows > 16) {
    const long n = (a.rows + 31) / 32 * ((outs + 3) / 4);
    if (units >= 2 && n <= cus && n >= 0.6 * cus) return launch_bf16<2>(a, 4, 2, s);
    if (outs >= 2 * cus && n > cus) {
      if (outs < 8 * cus) return launch_bf16<2>(a, a.rows <= 32 ? 4 : 8, 1, s);
      return a.rows <= 32 ? launch_bf16<2>(a, 8, 1, s) : launch_bf16<4>(a, 8, 1, s);
    }
    return some ? launch_bf16<1>(a, 4, n > cus ? 1 : four, s) : launch_bf16<1>(a, 2, two, s);
  }
  if (outs > 2 * cus && (units < 8 || outs >= 2.5 * cus)) return launch_bf16<1>(a, 4, four, s);
  return some ? launch_bf16<1>(a, 2, two, s) : launch_bf16<1>(a, 1, one, s);
}

}  // namespace hsa
