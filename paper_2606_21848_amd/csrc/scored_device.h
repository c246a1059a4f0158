// What the scored-attention kernels share: the seen ranges of query rows, and the
// score of a pair as a linear form of one number per pair.
#pragma once

#include <hip/hip_runtime.h>

#include "attn_tile.h"
#include "kl_device.h"
#include "kl_internal.h"

namespace kl {

constexpr float kScoredLog2e = 1.4426950408889634f;
constexpr float kScoredLn2 = 0.69314718055994531f;

// Lane permutation within rows of 16 lanes; lanes without a source get `none`.
template <int CTRL>
__device__ __forceinline__ int dpp_i32(int x, int none = 0) {
  return __builtin_amdgcn_update_dpp(none, x, CTRL, 0xF, 0xF, false);
}

// op over each row of 16 lanes (swapped neighbours, pairs, mirrored halves and rows); all
// of them get the result.
template <class Op>
__device__ __forceinline__ int row_reduce(int x, Op op) {
  x = op(x, dpp_i32<0xB1>(x));
  x = op(x, dpp_i32<0x4E>(x));
  x = op(x, dpp_i32<0x141>(x));
  return op(x, dpp_i32<0x140>(x));
}

// op over the wave, uniform.
template <class Op>
__device__ __forceinline__ int wave_reduce(int x, Op op) {
  x = row_reduce(x, op);
  return op(op(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)),
            op(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}

// The value rows [lo, hi) that query row i sees, within [0, N); an empty range is {0, 0}.
struct SeenRange {
  int lo, hi;
};
__device__ __forceinline__ SeenRange seen_range(const ScoredParams& p, int b, int i) {
  const size_t r = (size_t)b * p.N + i;
  const int lo = p.first ? max(p.first[r], 0) : 0;
  const int hi = p.last ? min(p.last[r], p.N) : (p.causal ? i + 1 : p.N);
  return lo < hi ? SeenRange{lo, hi} : SeenRange{0, 0};
}

// What a set of rows sees: rows outside [any_lo, any_hi) are seen by none of them, rows
// inside [all_lo, all_hi) by all. Of no rows, or of rows that see nothing, any is empty;
// a row that sees nothing leaves all empty.
struct SeenBounds {
  int any_lo = 0x7fffffff, any_hi = 0, all_lo = 0, all_hi = 0x7fffffff;
  __device__ __forceinline__ void add(SeenRange s) {
    if (s.lo < s.hi) {
      any_lo = min(any_lo, s.lo);
      any_hi = max(any_hi, s.hi);
    }
    all_lo = max(all_lo, s.lo);
    all_hi = min(all_hi, s.hi);
  }
  // Over each row of 16 lanes; all of them get the result.
  __device__ __forceinline__ void over_rows() {
    any_lo = row_reduce(any_lo, [](int a, int b) { return min(a, b); });
    any_hi = row_reduce(any_hi, [](int a, int b) { return max(a, b); });
    all_lo = row_reduce(all_lo, [](int a, int b) { return max(a, b); });
    all_hi = row_reduce(all_hi, [](int a, int b) { return min(a, b); });
  }
  // The same in scalar registers, once every lane holds the same.
  __device__ __forceinline__ void make_uniform() {
    any_lo = __builtin_amdgcn_readfirstlane(any_lo);
    any_hi = __builtin_amdgcn_readfirstlane(any_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  }
};

// x = cap tanh(z / cap) - slope dist in log2 units, from the dot product s (z = scale s).
// A pair is first turned into one number k with x = A k + C:
//   plain       k = s,                           A = scale log2 e,    C = 0
//   cap         k = 1 / (1 + exp(2 z / cap)),    A = -2 cap log2 e,   C = cap log2 e
//               (tanh(y) = 1 - 2 / (1 + exp(2 y)))
//   with bias   k = x itself,                    A = 1,               C = 0
// so that the shift by the row's maximum costs no operation of its own: the maximum
// is taken over k (its minimum where A < 0) and the weight is 2^(A k + (C - m)).
// d x / d z = 1 - tanh^2 = 4 k (1 - k) for the capped forms.
template <bool CAP, bool BIAS>
struct ScoreForm {
  static constexpr bool kFalling = CAP && !BIAS;  // a larger k is a smaller score
  float scale2;       // scale log2 e
  float cap2, twice;  // cap log2 e; 2 scale log2 e / cap
  __device__ __forceinline__ ScoreForm(float scale, float cap)
      : scale2(scale * kScoredLog2e), cap2(cap * kScoredLog2e),
        twice(CAP ? 2.f * scale * kScoredLog2e / cap : 0.f) {}
  __device__ __forceinline__ float A() const { return BIAS ? 1.f : CAP ? -2.f * cap2 : scale2; }
  __device__ __forceinline__ float C() const { return CAP && !BIAS ? cap2 : 0.f; }
  static __device__ __forceinline__ float unseen() { return kFalling ? INFINITY : -INFINITY; }
  // 1 / (1 + exp(2 z / cap)) for the capped forms.
  __device__ __forceinline__ float bent(float s) const {
    return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * twice));
  }
  // The key of a dot product; bias(x) gives x with its bias taken off, in log2 units.
  template <class Bias>
  __device__ __forceinline__ float key(float s, Bias bias) const {
    float k = s;
    if constexpr (CAP) k = bent(s);
    if constexpr (BIAS) k = bias(CAP ? fmaf(k, -2.f * cap2, cap2) : k * scale2);
    return k;
  }
  // The better of two keys.
  static __device__ __forceinline__ float best(float a, float b) {
    return kFalling ? fminf(a, b) : fmaxf(a, b);
  }
  // x - m from a key, with shift = C - m.
  __device__ __forceinline__ float shifted(float k, float shift) const {
    return BIAS ? k + shift : fmaf(A(), k, shift);
  }
};

__device__ __forceinline__ bool not_finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
}

// Two bf16 in a word, those that are not finite replaced by zero.
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) |
         ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) unsigned char lds_u8;

// Instruction classes of __builtin_amdgcn_sched_group_barrier.
constexpr int kSchedMfma = 0x008, kSchedDsRead = 0x100;

__device__ __forceinline__ bf16x8_t finite_or_zero(bf16x8_t v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int x = 0; x < 4; ++x) w[x] = finite_or_zero(w[x]);
  return __builtin_bit_cast(bf16x8_t, w);
}

__device__ __forceinline__ bf16x8_t pack8(f32x4_t a, f32x4_t b) {
  return __builtin_bit_cast(bf16x8_t, u32x4{pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]),
                                            pack2(b[2], b[3])});
}

// One 16-byte row fragment at an LDS address.
__device__ __forceinline__ bf16x8_t lds_rows(int at) {
  return *(const __attribute__((address_space(3))) bf16x8_t*)(uintptr_t)(uint32_t)at;
}

// One 16-column block of 32 rows, transposed: rows 4 grp .. + 3 and 16 + 4 grp .. + 3 of
// this lane's column.
template <int ROW>
__device__ __forceinline__ bf16x8_t lds_columns(int at) {
  const lds_u8* src = (const lds_u8*)(uintptr_t)(uint32_t)at;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)src);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(src + 16 * ROW));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A workgroup's (4 waves) copies of 64-row tiles of a [rows, ...] bf16 matrix, D columns
// from its base, into an AttnTile<D, 64>: copy c of a wave fills the tile rows
// (4 c + wave) RPC .. + RPC - 1; rows past the end are copies of the last one.
template <int D>
struct TileCopy {
  using T = AttnTile<D, 64>;
  static constexpr int RPC = 1024 / T::ROW, COPIES = T::COPIES;
  uint32_t chunk;  // of the lane's row, the same for every copy: they lie 16 rows or 32 apart,
                   // which is a whole period of the swizzle
  uint32_t lane_row;
  __device__ __forceinline__ TileCopy(int wave, int lane, size_t row_bytes)
      : chunk((uint32_t)(T::swz(wave * RPC + lane / T::CHUNKS, lane % T::CHUNKS) * 16)),
        lane_row((uint32_t)(lane / T::CHUNKS) * (uint32_t)row_bytes) {}
  __device__ __forceinline__ void issue(const unsigned char* g, size_t row_bytes, int row0, int n_rows,
                                        int wave, int lane, uint32_t lds) const {
    if (row0 + 64 <= n_rows) {
      const unsigned char* base = g + (size_t)row0 * row_bytes;
#pragma unroll
      for (int c = 0; c < COPIES; ++c)
        copy_to_lds(base + (size_t)((c * 4 + wave) * RPC) * row_bytes, lane_row + chunk,
                    lds + (c * 4 + wave) * 1024);
    } else {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) {
        const int r0 = row0 + (c * 4 + wave) * RPC, r0c = min(r0, n_rows - 1);
        const int rl = min(r0 + lane / T::CHUNKS, n_rows - 1) - r0c;
        copy_to_lds(g + (size_t)r0c * row_bytes, (uint32_t)(rl * row_bytes) + chunk,
                    lds + (c * 4 + wave) * 1024);
      }
    }
  }
};

// Which head and query tile a workgroup of a 1-d grid takes. Groups vary fastest, then
// a group's heads: consecutive workgroups go to different XCDs, so where G is a multiple
// of 8 the heads that read one group's values share an XCD's L2. The last query tiles
// (under the causal mask the heaviest) start first.
struct HeadTile {
  int h, g, b, qt;
  __device__ __forceinline__ HeadTile(const ScoredParams& p, int rows) {
    const int R = p.H / p.G, tiles = (p.N + rows - 1) / rows;
    g = blockIdx.x % p.G;
    h = g * R + blockIdx.x / p.G % R;
    const unsigned rest = blockIdx.x / p.H;
    b = rest % p.B;
    qt = tiles - 1 - rest / p.B;
  }
};

constexpr float kLazy = 8.f;  // a softmax reference moves when a score exceeds it by 2^8

// The online softmax of QB 16-query blocks over NB 16-row blocks of values: sc holds
// the dot products on entry (lane: query fr of block qb, rows 16 kb + 4 grp + r of the
// tile) and the weights on return. `edge` (uniform): some row is not seen by some query,
// as unseen(qb, kb, r) tells; bias(x, qb, kb, r) takes a pair's bias off; returns whether a
// pair that is not seen has a product that is not finite (uniform). Its value row is then
// not finite, and 0 times it would not be either: the caller takes the values that are not finite as zeros, and a query that
// sees such a product gets NaN as its score here, and with it as its result.
template <int D, int NB, int QB, class Form, class Unseen, class Bias>
__device__ __forceinline__ bool soften(const Form& form, f32x4_t (&sc)[NB][QB], f32x4_t (&o)[D / 16][QB],
                                       float (&m)[QB], float (&l)[QB], bool edge, Unseen unseen, Bias bias) {
  bool bad = false;
  if (edge) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          bad |= unseen(qb, kb, r) & not_finite(sc[kb][qb][r]);
    bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (bad) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            sc[kb][qb][r] = not_finite(sc[kb][qb][r]) ? __builtin_nanf("") : sc[kb][qb][r];
    }
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[kb][qb][r] = form.key(sc[kb][qb][r], [&](float x) { return bias(x, qb, kb, r); });
  if (edge) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          sc[kb][qb][r] = unseen(qb, kb, r) ? Form::unseen() : sc[kb][qb][r];
  }
  float top[QB];  // this lane's best score per query
  bool grow = false;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    float k = sc[0][qb][0];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) k = Form::best(k, sc[kb][qb][r]);
    top[qb] = fmaf(form.A(), k, form.C());
    grow |= top[qb] > m[qb] + kLazy;
  }
  if (__builtin_amdgcn_ballot_w64(grow)) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float t = fmaxf(top[qb], __shfl_xor(top[qb], 16));
      t = fmaxf(t, __shfl_xor(t, 32));
      const float mn = t > m[qb] + kLazy ? t : m[qb];
      const float alpha = m[qb] == -INFINITY ? 0.f : fast_exp2(m[qb] - mn);
      l[qb] *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i][qb] *= alpha;
      m[qb] = mn;
    }
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float shift = form.C() - (m[qb] == -INFINITY ? 0.f : m[qb]);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[kb][qb][r] = fast_exp2(form.shifted(sc[kb][qb][r], shift));
      l[qb] += (sc[kb][qb][0] + sc[kb][qb][1]) + (sc[kb][qb][2] + sc[kb][qb][3]);
    }
  }
  return bad;
}

// Merge of the NW waves of a workgroup, each with partial results of the same 16 QB rows:
// the sums are scaled to the rows' common reference and added in wave order. A wave that
// saw nothing of a row has reference -inf (and sums of zero). Every wave's place of LDS
// at ring0 + wave * stride holds its results.
template <int D, int QB, int NW>
struct WaveMerge {
  float (*ml)[16 * QB][2];
  uint32_t ring0, stride;
  int wave, fr, grp;
  __device__ __forceinline__ WaveMerge(float (*s_ml)[16 * QB][2], uint32_t ring0_, uint32_t stride_, int wave_,
                                       int fr_, int grp_)
      : ml(s_ml), ring0(ring0_), stride(stride_), wave(wave_), fr(fr_), grp(grp_) {}
  __device__ __forceinline__ float top(int row) const {
    float x = ml[0][row][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) x = fmaxf(x, ml[w][row][0]);
    return x;
  }
  // l: this lane's part of the weight sums.
  __device__ __forceinline__ void put(const float (&m)[QB], const float (&l)[QB], const f32x4_t (&o)[D / 16][QB]) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's tiles have been read
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float sum = l[qb] + __shfl_xor(l[qb], 16);
      sum += __shfl_xor(sum, 32);
      if (grp == 0) {
        ml[wave][qb * 16 + fr][0] = m[qb];
        ml[wave][qb * 16 + fr][1] = sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float mm = top(qb * 16 + fr), f = fast_exp2(m[qb] - (mm == -INFINITY ? 0.f : mm));
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
        WaveSums<D>::put(ring0 + wave * stride, qb * 16 + fr, 4 * db + grp, o[db][qb] * f);
    }
    __syncthreads();
  }
  // Four columns of a row, its reference and its weight sum.
  __device__ __forceinline__ f32x4_t get(int row, int piece, float& mm, float& sum) const {
    mm = top(row);
    const float ms = mm == -INFINITY ? 0.f : mm;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += ml[w][row][1] * fast_exp2(ml[w][row][0] - ms);
    return WaveSums<D>::template get<NW>(ring0, stride, row, piece);
  }
};

}  // namespace kl
