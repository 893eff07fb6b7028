// Where the workgroups of a packed attention launch find their rows.
//
// With grouped heads the G query heads of one key/value head see the same keys,
// so the rows of a tile are (query, head of the group) pairs, R = query * G +
// head: a tile of 256 rows at G = 4 spans 64 queries, its keys are
// loaded once for the four heads, and a causal tile wastes half of 64 keys at
// its end, not half of 256.
#pragma once

#include "seq_common.h"

#include <algorithm>
#include <cmath>

namespace hsa {

struct SeqTile {
  int q0, len_q, k0, len_k;  // rows of the sequence
  int tile;                  // its tile of this workgroup
};

// Heads and tiles over the XCDs: workgroup L runs on XCD L % 8. The heads that
// one XCD works on are those congruent to it mod c = gcd(8, kv_heads), and the
// 8 / c XCDs of a head take its tiles in turn, so that whatever kv_heads is
// every XCD gets as much of a causal sequence's long tiles as of its short ones, and a
// head's keys pass through as few L2s as that allows. An XCD takes its heads
// one after the other, or, where the keys and values of all of them fit its L2 of 4 MB, in
// turn, tile by tile, so that every head's longest tiles come first. One causal prompt, one after the other
// and in turn, us (MB: keys and values of an XCD's heads):
//   40 heads x 64   1000 tokens (1.2 MB)  23.4  18.4    1500 (1.8)  28.8  24.4
//   40 heads x 128  1000 (2.4)            30.1  30.1    2500 (6.1)  95.3  74.9    8000 (19.5)  660  617
//   12 heads x 64   1000 (0.7)            15.6  12.8    4000 (2.9)  67.2  51.6
// Without a mask the two are within 2%, in turn 1% slower at 16000 tokens. So the limit is that of the
// L2, not of what a causal prompt would gain beyond it.
struct PackedGrid {
  int share;   // XCDs per head
  int per;     // tiles of one head on one XCD, at most
  int heads;   // heads of an XCD
  int turns;   // heads in turn
  int groups;  // workgroups
};
inline PackedGrid packed_grid(const PackedArgs& a, int rows, int row_bytes) {
  int c = 8;
  while (a.kv_heads % c) c >>= 1;
  const long tiles = (long)a.n_q * a.group / rows + a.n_seqs;  // sum of ceil(rows of a sequence / rows of a tile), at most
  const long share = 8 / c, per = (tiles + share - 1) / share, heads = a.kv_heads / c;
  const long groups = per * heads * 8;
  const bool turns = heads * a.n_kv * 2 * row_bytes <= 3L << 20;
  return {(int)share, (int)per, (int)heads, turns, groups < INT32_MAX ? (int)groups : -1};
}
__device__ __forceinline__ void packed_place(const PackedGrid& g, int& head, int& tile) {
  const int c = kXcds / g.share;
  const int xcd = blockIdx.x % kXcds, slot = blockIdx.x / kXcds;
  const int n = g.turns ? g.heads : g.per, x = slot / n, y = slot - x * n;
  head = xcd % c + c * (g.turns ? y : x);
  tile = xcd / c + g.share * (g.turns ? x : y);
}

// Rows of sequence `s`, inside [0, n) whatever the offsets hold.
__device__ __forceinline__ void seq_rows(const int32_t* cu, int s, int n, int& from, int& to) {
  from = min(max(cu[s], 0), n);
  to = min(max(cu[s + 1], from), n);
}

// Tile `idx` of the batch; false for one that no sequence has. Within a sequence
// the last tile comes first (under a causal mask the longest). Called by whole
// waves; the result is the same in every lane.
//   Up to 64 sequences, one to a lane: in the order of their tiles, the longest
//   first, so that what runs last is short.
//   More: as they are, sequence s from tile floor(cu_q[s] G / ROWS) + s on, which leaves
//   each at least its tiles; found by probing 64 sequences at a time.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const PackedArgs& a, int idx, SeqTile& t) {
  const int lane = threadIdx.x & (kWave - 1);
  if (a.n_seqs <= kWave) {
    int q0 = 0, q1 = 0, k0 = 0, k1 = 0;
    if (lane < a.n_seqs) {
      seq_rows(a.cu_q, lane, a.n_q, q0, q1);
      seq_rows(a.cu_kv, lane, a.n_kv, k0, k1);
    }
    const int tiles = (int)(((long)(q1 - q0) * a.group + ROWS - 1) / ROWS);
    int from = 0;  // tiles before this lane's sequence
    for (int i = 0; i < a.n_seqs; ++i) {
      const int n = __builtin_amdgcn_readlane(tiles, i);
      from += n > tiles || (n == tiles && i < lane) ? n : 0;
    }
    const unsigned long hit = __ballot(from <= idx && idx < from + tiles);
    if (!hit) return false;
    const int l = __builtin_ctzl(hit);
    t.q0 = __builtin_amdgcn_readlane(q0, l);
    t.len_q = __builtin_amdgcn_readlane(q1, l) - t.q0;
    t.k0 = __builtin_amdgcn_readlane(k0, l);
    t.len_k = __builtin_amdgcn_readlane(k1, l) - t.k0;
    t.tile = __builtin_amdgcn_readlane(tiles, l) - 1 - (idx - __builtin_amdgcn_readlane(from, l));
    return true;
  }
  auto first = [&](int s) { return (int)((long)min(max(a.cu_q[s], 0), a.n_q) * a.group / ROWS) + s; };
  int lo = 0;  // the last sequence whose first tile is at most idx is one of lo .. lo+n-1
  for (int n = a.n_seqs; n > 1;) {
    const int step = (n + kWave - 1) / kWave;
    const unsigned long below = __ballot(lane * step < n && first(lo + min(lane * step, n - 1)) <= idx);
    if (!below) return false;
    const int l = kWave - 1 - __builtin_clzl(below);
    lo += l * step;
    n = min(step, n - l * step);
  }
  int q1, k1;
  seq_rows(a.cu_q, lo, a.n_q, t.q0, q1);
  seq_rows(a.cu_kv, lo, a.n_kv, t.k0, k1);
  t.q0 = __builtin_amdgcn_readfirstlane(t.q0);
  t.len_q = __builtin_amdgcn_readfirstlane(q1) - t.q0;
  t.k0 = __builtin_amdgcn_readfirstlane(t.k0);
  t.len_k = __builtin_amdgcn_readfirstlane(k1) - t.k0;
  const int tiles = (int)(((long)t.len_q * a.group + ROWS - 1) / ROWS);
  t.tile = tiles - 1 - (idx - __builtin_amdgcn_readfirstlane(first(lo)));
  return t.tile >= 0 && t.tile < tiles;
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

// adds to 4 channels of a row that has a finite score the values of keys from .. end-1 that are not finite
__device__ __forceinline__ void add_odd(f32x4& sum, const bf16* v, long stride, int from, int end) {
  for (int n = from; n < end; ++n)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float x = (float)v[n * stride + u];
      if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) sum[u] += x;
    }
}

// bf16, 128 or 256 rows per workgroup, for 64- and 128-wide heads (packed_attention_large.hip)
hipError_t launch_packed_attention_large(const PackedArgs& a, int head_dim, hipStream_t s);
// Estimated time of a launch with tiles of `rows` rows and workgroups of `waves` waves (us,
// MI355X), from the means of the batch's lengths, which are all the host knows: a fixed
// part, and the tiles' share of a CU (each a start and its 32-key blocks; up to 4 tiles
// to a CU count whole) or one tile's chain of blocks, whichever is longer. Means hide a long sequence
// among many short ones: 4500 tokens and 255 of one, 8/8 heads of 128, take 200 us with a causal
// mask and 359 without one in the 16-row tiles that their mean asks for, 95 and 114 in those of 256;
// with 63 of one, 98 and 103 in the right ones.
struct PackedCost {
  int rows, waves;
  double fixed, tile, block, chain;
};
// The tile forced for this thread's launches (packed_tile.h); rows 0: none. 128 and 256 rows both
// mean the large kernel, which has one of them for either width.
struct PackedTile {
  int rows, waves;
  bool is(const PackedCost& c) const { return rows == c.rows && waves == c.waves; }
  bool large() const { return (rows == 128 && waves == 4) || (rows == 256 && waves == 8); }
};
PackedTile& packed_tile();
// The cheapest of N shapes; NULL where one is forced that is none of them.
template <int N>
inline const PackedCost* packed_choice(const PackedArgs& a, const PackedCost (&costs)[N]) {
  const PackedTile forced = packed_tile();
  if (forced.rows) {
    for (const PackedCost& c : costs)
      if (forced.is(c) || (forced.large() && c.rows >= 128)) return &c;
    return nullptr;
  }
  const double seqs = a.n_seqs, len_q = a.n_q / seqs, len_k = a.n_kv / seqs;
  const double blocks = std::max(0.0, len_k - (a.causal ? len_q / 2 : 0.0)) / 32;
  const PackedCost* best = &costs[0];
  double least = 0.0;
  for (const PackedCost& c : costs) {
    const double tiles = seqs * std::ceil(len_q * a.group / c.rows) * a.kv_heads;
    const double each = tiles / compute_units();
    const double us = c.fixed + std::max((each > 4 ? each : std::ceil(each)) * (c.tile + c.block * blocks),
                                         c.tile + c.chain * len_k / 32);
    if (&c == &costs[0] || us < least) {
      best = &c;
      least = us;
    }
  }
  return best;
}

hipError_t launch_packed_attention_f32(const PackedArgs& a, int head_dim, hipStream_t s);

}  // namespace hsa
