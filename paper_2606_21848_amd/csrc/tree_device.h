// The work split of the drafted-token decode, which its kernels derive from the lengths
// on the device: the rows of every sequence (cached and drafted) are cut into chunks of
// `per` 32-row tiles, chunk after chunk and sequence after sequence. A sequence of one
// chunk is written by the workgroups that hold it; the others leave partial results that
// a merge kernel joins in chunk order.
#pragma once

#include <hip/hip_runtime.h>

#include "kl_internal.h"

namespace kl {

constexpr int kTreeTile = 32;  // rows per tile

struct TreeSpan {
  int b, s, S;     // sequence, chunk of it, its chunks
  int first;       // its first chunk among all
  int n, rows;     // rows cached before the draft, rows in all
  int tile0, tiles;
};

__device__ __forceinline__ int tree_cached(const TreeParams& p, int b) {
  const int cap = p.paged ? p.max_blocks << p.block_shift : p.L_max;
  return min(max(((const __attribute__((address_space(4))) int*)p.lengths)[b], 0), cap);
}
__device__ __forceinline__ int tree_rows(const TreeParams& p, int n) {
  const int cap = p.paged ? p.max_blocks << p.block_shift : p.L_max;
  return min(n + p.T, cap);
}
__device__ __forceinline__ int tree_lane_tiles(const TreeParams& p, int b) {
  if (b >= p.B) return 0;
  const int cap = p.paged ? p.max_blocks << p.block_shift : p.L_max;
  const int n = min(max(p.lengths[b], 0), cap);
  // A sequence has one chunk at least, whose workgroups write its zero rows.
  return max((tree_rows(p, n) + kTreeTile - 1) / kTreeTile, 1);
}

__device__ __forceinline__ long wave_sum(long x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// Tiles per chunk: the fewest that give at most p.chunks chunks, and p.least at least
// (with more than 64 sequences, or not many fewer than chunks, an even share of all
// tiles, which gives at most B chunks more).
__device__ __forceinline__ int tree_per(const TreeParams& p, int lane) {
  long total = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) total += wave_sum((long)tree_lane_tiles(p, b0 + lane));
  int per = max((int)((total + p.chunks - 1) / p.chunks), p.least);
  if (p.B <= 64 && 2 * p.B <= p.chunks) {
    const int n = tree_lane_tiles(p, lane);
    int fits = 2 * per;  // sum ceil(n / 2 per) <= chunks / 2 + B
    int lo = per;
    while (lo < fits) {
      const int mid = (lo + fits) / 2;
      if (wave_sum((n + mid - 1) / mid) <= p.chunks) fits = mid;
      else lo = mid + 1;
    }
    per = fits;
  }
  return __builtin_amdgcn_readfirstlane(per);
}

// The chunk `c` of all (want_b < 0), or the first chunk of sequence want_b; false when
// there are not that many. Uniform over the wave.
__device__ __forceinline__ bool tree_span(const TreeParams& p, int lane, int c, int want_b, TreeSpan& t) {
  const int per = tree_per(p, lane);
  int before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int S = (tree_lane_tiles(p, b0 + lane) + per - 1) / per;
    int pre = S;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(pre, o);
      if (lane >= o) pre += x;
    }
    const int all = __builtin_amdgcn_readlane(pre, 63);
    const uint64_t hit = want_b < 0 ? __builtin_amdgcn_ballot_w64(before + pre > c)
                                    : (want_b < b0 + 64 ? 1ull << (want_b - b0) : 0);
    if (hit) {
      const int at = __builtin_ctzll(hit);
      t.b = b0 + at;
      t.S = __builtin_amdgcn_readlane(S, at);
      t.first = before + __builtin_amdgcn_readlane(pre, at) - t.S;
      t.s = want_b < 0 ? c - t.first : 0;
      t.n = tree_cached(p, t.b);
      t.rows = tree_rows(p, t.n);
      t.tile0 = t.s * per;
      t.tiles = min((t.rows + kTreeTile - 1) / kTreeTile - t.tile0, per);
      return true;
    }
    before += all;
  }
  return false;
}

// What drafted token t sees of the draft, as a word without bits past T; its depth.
__device__ __forceinline__ uint64_t tree_word(const TreeParams& p, int b, int t) {
  const uint64_t all = p.T == 64 ? ~0ull : (1ull << p.T) - 1;
  return p.tree ? p.tree[(size_t)b * p.T + t] & all : (2ull << t) - 1;
}
__device__ __forceinline__ int tree_depth(uint64_t word, int t) { return __popcll(word & ~(1ull << t)); }

// Where chunk c leaves row m of group g: its weighted sums [D], and its reference (log2
// units) and weight sum.
__device__ __forceinline__ float* tree_part(const TreeParams& p, int c, int g, int m) {
  return p.part + (((size_t)c * p.G + g) * p.T * (p.H / p.G) + m) * p.D;
}
__device__ __forceinline__ float* tree_part_ml(const TreeParams& p, int c, int g, int m) {
  return p.part_ml + (((size_t)c * p.G + g) * p.T * (p.H / p.G) + m) * 2;
}

}  // namespace kl
