// The work split of the drafted-token decode, which its kernels derive from the lengths
// on the device. A sequence's rows, cached and drafted, are 32-row tiles.
//  - Shared (p.per == 0): the tiles of all sequences, one after another, are cut into
//    p.chunks even pieces, whatever the spread of lengths; a workgroup walks its piece
//    sequence by sequence.
//  - Fixed (p.per > 0, few sequences): piece s of p.chunks pieces of each sequence is its
//    tiles from s p.per on; nothing has to be summed first.
// A sequence inside one piece is written by its workgroups; the others leave partial
// results in slots of their own that a merge kernel joins in order.
#pragma once

#include <hip/hip_runtime.h>

#include "kl_internal.h"
#include "scored_device.h"

namespace kl {

constexpr int kTreeTile = 32;  // rows per tile

__device__ __forceinline__ int tree_capacity(const TreeParams& p) {
  return p.paged ? p.max_blocks << p.block_shift : p.L_max;
}
// Rows cached before the draft, and rows in all.
__device__ __forceinline__ int tree_cached(const TreeParams& p, int b) {
  return min(max(((const __attribute__((address_space(4))) int*)p.lengths)[b], 0), tree_capacity(p));
}
__device__ __forceinline__ int tree_rows(const TreeParams& p, int n) { return min(n + p.T, tree_capacity(p)); }
// Tiles of a sequence: one at least, whose workgroups write its zero rows.
__device__ __forceinline__ int tree_tiles(int rows) { return max((rows + kTreeTile - 1) / kTreeTile, 1); }
__device__ __forceinline__ int tree_lane_tiles(const TreeParams& p, int b) {
  if (b >= p.B) return 0;
  return tree_tiles(tree_rows(p, min(max(p.lengths[b], 0), tree_capacity(p))));
}

__device__ __forceinline__ int wave_sum(int x) {  // uniform
  return wave_reduce(x, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int wave_prefix(int x, int lane) {  // inclusive
  x += dpp_i32<0x111>(x);  // by 1, 2, 4 and 8 lanes within rows of 16
  x += dpp_i32<0x112>(x);
  x += dpp_i32<0x114>(x);
  x += dpp_i32<0x118>(x);
  const int a = __builtin_amdgcn_readlane(x, 15), b = a + __builtin_amdgcn_readlane(x, 31),
            c = b + __builtin_amdgcn_readlane(x, 47);
  return x + (lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? b : c);
}

// The shared split: tiles per piece, and whether every sequence starts a piece of its own.
// A workgroup's second sequence costs it the latencies of a start and a merge, some 5 us,
// the time of a dozen tiles: short pieces are kept apart (6 sequences of 5 to 1500 rows,
// fp32: 15.8 us across them, 12.6 apart).
struct TreeShare {
  int per, total;
  bool apart;
  // Tiles of a sequence of n, with the idle ones behind it that end its last piece.
  __device__ __forceinline__ int padded(int n) const { return apart ? (n + per - 1) / per * per : n; }
};
constexpr int kShortPiece = 16;
__device__ __forceinline__ TreeShare tree_share(const TreeParams& p, int lane) {
  TreeShare s;
  s.total = 0;
  int n = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    n = tree_lane_tiles(p, b0 + lane);
    s.total += wave_sum(n);
  }
  s.per = max((s.total + p.chunks - 1) / p.chunks, p.least);
  s.apart = p.B <= 64 && 2 * p.B <= p.chunks && s.per <= kShortPiece;
  if (s.apart) {
    // At twice the even share there are at most chunks / 2 + B pieces: this ends.
    int pieces = wave_sum((n + s.per - 1) / s.per);
    while (pieces > p.chunks) pieces = wave_sum((n + ++s.per - 1) / s.per);
    s.total = pieces * s.per;
  }
  return s;
}

struct TreeSeg {
  int b, n, rows;     // sequence, rows cached before its draft, rows in all
  int tile0, tiles;   // the piece's tiles of it
  int slot;           // where partial results go
  bool whole;         // all of its tiles
};

// The segments of piece c; uniform over the wave.
struct TreeWalk {
  int c, b, b0, tiles_of_lane, off, left;
  TreeShare share;
  __device__ __forceinline__ TreeWalk(const TreeParams& p, int lane, int c_) : c(c_), b(0), b0(0), off(0) {
    if (p.per > 0) {
      b = c / p.chunks;
      left = 1;
      return;
    }
    share = tree_share(p, lane);
    const int from = c * share.per;
    left = min(share.per, share.total - from);
    if (left <= 0) return;
    int before = 0;
    for (;; b0 += 64) {
      tiles_of_lane = share.padded(tree_lane_tiles(p, b0 + lane));
      const int pre = wave_prefix(tiles_of_lane, lane);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(before + pre > from);
      if (hit) {
        const int at = __builtin_ctzll(hit);
        b = b0 + at;
        off = from - (before + __builtin_amdgcn_readlane(pre, at) - __builtin_amdgcn_readlane(tiles_of_lane, at));
        return;
      }
      before += __builtin_amdgcn_readlane(pre, 63);
    }
  }
  __device__ __forceinline__ bool next(const TreeParams& p, int lane, TreeSeg& s) {
    if (left <= 0) return false;
    s.b = b;
    s.n = tree_cached(p, b);
    s.rows = tree_rows(p, s.n);
    const int real = (s.rows + kTreeTile - 1) / kTreeTile;
    if (p.per > 0) {
      left = 0;
      s.tile0 = (c - b * p.chunks) * p.per;
      if (s.tile0 > 0 && s.tile0 >= real) return false;
      s.tiles = min(real - s.tile0, p.per);
      s.whole = real <= p.per;
      s.slot = c;
      return true;
    }
    const int all = __builtin_amdgcn_readlane(tiles_of_lane, b - b0), take = min(all - off, left);
    s.tile0 = off;
    s.tiles = min(real - off, take);
    s.whole = take == all;
    s.slot = c + b;  // along the pieces c and b never fall, and one of them grows
    left -= take;
    off = 0;
    if (++b == b0 + 64) {
      b0 += 64;
      tiles_of_lane = share.padded(tree_lane_tiles(p, b0 + lane));
    }
    return true;
  }
};

// The slots that hold sequence b's partial results: `count` from `first` on; one when the
// sequence was written directly.
__device__ __forceinline__ int tree_slots(const TreeParams& p, int lane, int b, int& first) {
  if (p.per > 0) {
    first = b * p.chunks;
    return (tree_tiles(tree_rows(p, tree_cached(p, b))) + p.per - 1) / p.per;
  }
  const TreeShare share = tree_share(p, lane);
  const int per = share.per;
  int before = 0, b0 = 0;
  for (; b0 + 64 <= b; b0 += 64) before += wave_sum(share.padded(tree_lane_tiles(p, b0 + lane)));
  const int n = share.padded(tree_lane_tiles(p, b0 + lane)), pre = wave_prefix(n, lane);
  const int end = before + __builtin_amdgcn_readlane(pre, b - b0), from = end - __builtin_amdgcn_readlane(n, b - b0);
  first = from / per + b;
  return (end - 1) / per - from / per + 1;
}

// What drafted token t sees of the draft, as a word without bits past T; its depth.
__device__ __forceinline__ uint64_t tree_word(const TreeParams& p, int b, int t) {
  const uint64_t all = p.T == 64 ? ~0ull : (1ull << p.T) - 1;
  return p.tree ? p.tree[(size_t)b * p.T + t] & all : (2ull << t) - 1;
}
__device__ __forceinline__ int tree_depth(uint64_t word, int t) { return __popcll(word & ~(1ull << t)); }

// Row m of group g in slot c: its weighted sums [D], and its reference (log2 units) and
// weight sum.
__device__ __forceinline__ float* tree_part(const TreeParams& p, int c, int g, int m) {
  return p.part + (((size_t)c * p.G + g) * p.T * (p.H / p.G) + m) * p.D;
}
__device__ __forceinline__ float* tree_part_ml(const TreeParams& p, int c, int g, int m) {
  return p.part_ml + (((size_t)c * p.G + g) * p.T * (p.H / p.G) + m) * 2;
}

}  // namespace kl
