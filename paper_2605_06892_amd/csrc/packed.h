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

// Tile `idx` of the batch: the sequences in order, and within a sequence the
// last tile first (under a causal mask the longest). False past the last one.
// Whatever the offsets hold, the rows are inside [0, n_q) and [0, n_kv).
// Called by whole waves; the result is the same in every lane.
__device__ __forceinline__ bool find_tile(const PackedArgs& a, int idx, int rows, SeqTile& t) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    const int s = s0 + lane;
    int q0 = 0, q1 = 0;
    if (s < a.n_seqs) {
      q0 = min(max(a.cu_q[s], 0), a.n_q);
      q1 = min(max(a.cu_q[s + 1], q0), a.n_q);
    }
    const int tiles = (int)(((long)(q1 - q0) * a.group + rows - 1) / rows);
    int upto = tiles;  // tiles of the sequences s0 .. s
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned long hit = __ballot(idx < upto);
    if (hit) {
      const int l = __builtin_ctzl(hit);
      t.q0 = __builtin_amdgcn_readlane(q0, l);
      t.len_q = __builtin_amdgcn_readlane(q1, l) - t.q0;
      const int n = __builtin_amdgcn_readlane(tiles, l);
      t.tile = n - 1 - (idx - (__builtin_amdgcn_readlane(upto, l) - n));
      if (t.tile < 0 || t.tile >= n) return false;  // offsets in no order
      t.k0 = min(max(a.cu_kv[s0 + l], 0), a.n_kv);
      t.len_k = min(max(a.cu_kv[s0 + l + 1], t.k0), a.n_kv) - t.k0;
      return true;
    }
    idx -= __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return false;
}

// keys that query i of the sequence sees (at most 0: none)
__device__ __forceinline__ int keys_seen(const PackedArgs& a, const SeqTile& t, int i) {
  return a.causal ? min(t.len_k, i + 1 + t.len_k - t.len_q) : t.len_k;
}

hipError_t launch_packed_attention_f32(const PackedArgs& a, int head_dim, hipStream_t s);

}  // namespace hsa
