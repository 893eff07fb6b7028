// Where the workgroups of a packed attention launch find their rows.
//
// With grouped heads the G query heads of one key/value head see the same keys,
// so the rows of a tile are (query, head of the group) pairs, R = query * G +
// head: a tile of 256 rows at G = 4 spans 64 queries, its keys are
// loaded once for the four heads, and a causal tile wastes half of 64 keys at
// its end, not half of 256.
#pragma once

#include "seq_common.h"

namespace hsa {

struct SeqTile {
  int q0, len_q, k0, len_k;  // rows of the sequence
  int tile;                  // its tile of this workgroup
};

// Heads and tiles over the XCDs: workgroup L runs on XCD L % 8. The heads that
// one XCD works on are those congruent to it mod c = gcd(8, kv_heads), and the
// 8 / c XCDs of a head take its tiles in turn, so that whatever kv_heads is
// every XCD gets as much of a causal sequence's long tiles as of its short ones, and a
// head's keys pass through as few L2s as that allows.
struct PackedGrid {
  int share;   // XCDs per head
  int per;     // tiles of one head on one XCD, at most
  int groups;  // workgroups
};
inline PackedGrid packed_grid(int n_q, int n_seqs, int kv_heads, int group, int rows) {
  int c = 8;
  while (kv_heads % c) c >>= 1;
  const long tiles = (long)n_q * group / rows + n_seqs;  // sum of ceil(rows of a sequence / rows of a tile), at most
  const long share = 8 / c, per = (tiles + share - 1) / share;
  const long groups = per * kv_heads * share;
  return {(int)share, (int)per, groups < INT32_MAX ? (int)groups : -1};
}
__device__ __forceinline__ void packed_place(const PackedGrid& g, int kv_heads, int& head, int& tile) {
  const int c = kXcds / g.share;
  const int xcd = blockIdx.x % kXcds, slot = blockIdx.x / kXcds;
  const int i = slot / g.per;  // the i-th head of this XCD, all its tiles before the next head's
  head = xcd % c + c * i;
  tile = xcd / c + g.share * (slot - i * g.per);
}

// Tile `idx` of the batch: the sequences one after the other, and within a
// sequence the last tile first (under a causal mask the longest). Up to 64 sequences
// come in the order of their tiles, the longest first, so that what runs last is
// short; more come as they are. False past the last tile. Whatever the offsets hold, the rows are
// inside [0, n_q) and [0, n_kv). Called by whole waves; the result is the same in every lane.
__device__ __forceinline__ bool find_tile(const PackedArgs& a, int idx, int rows, SeqTile& t) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    const int s = s0 + lane;
    int q0 = 0, q1 = 0, k0 = 0, k1 = 0;
    if (s < a.n_seqs) {
      q0 = min(max(a.cu_q[s], 0), a.n_q);
      q1 = min(max(a.cu_q[s + 1], q0), a.n_q);
      k0 = min(max(a.cu_kv[s], 0), a.n_kv);
      k1 = min(max(a.cu_kv[s + 1], k0), a.n_kv);
    }
    const int tiles = (int)(((long)(q1 - q0) * a.group + rows - 1) / rows);
    int from = 0, all = 0;  // tiles before this lane's sequence, and of the 64
    if (a.n_seqs <= kWave) {
      for (int i = 0; i < a.n_seqs; ++i) {
        const int n = __builtin_amdgcn_readlane(tiles, i);
        from += n > tiles || (n == tiles && i < lane) ? n : 0;
        all += n;
      }
    } else {
      all = tiles;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int y = __shfl_up(all, o);
        if (lane >= o) all += y;
      }
      from = all - tiles;
      all = __builtin_amdgcn_readlane(all, kWave - 1);
    }
    const unsigned long hit = __ballot(from <= idx && idx < from + tiles);
    if (hit) {
      const int l = __builtin_ctzl(hit);
      t.q0 = __builtin_amdgcn_readlane(q0, l);
      t.len_q = __builtin_amdgcn_readlane(q1, l) - t.q0;
      t.tile = __builtin_amdgcn_readlane(tiles, l) - 1 - (idx - __builtin_amdgcn_readlane(from, l));
      t.k0 = __builtin_amdgcn_readlane(k0, l);
      t.len_k = __builtin_amdgcn_readlane(k1, l) - t.k0;
      return true;
    }
    idx -= all;
  }
  return false;
}

// keys that query i of the sequence sees (at most 0: none)
__device__ __forceinline__ int keys_seen(const PackedArgs& a, const SeqTile& t, int i) {
  return a.causal ? min(t.len_k, i + 1 + t.len_k - t.len_q) : t.len_k;
}

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

// bf16, 256 rows per workgroup (packed_attention_large.hip)
hipError_t launch_packed_attention_large(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_packed_attention_f32(const PackedArgs& a, int head_dim, hipStream_t s);

}  // namespace hsa
