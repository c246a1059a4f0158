// Scored keyless attention and drafted-token decode in fp32, on the matrix cores
// (v_mfma_f32_16x16x4_f32: fp32 products and sums). As in the unscored fp32 kernels, a
// workgroup owns one 16-row block (queries for the output and dQ~, values for dV, query
// rows of a group for a draft) and its waves share the 16-row blocks that it meets, each
// with a private LDS tile, until their partial results are merged in wave order: a 16 x
// 16 block of scores and its weighted sum cost D / 2 products of 32 cycles, beside which
// an accurate tanh (the library's, a few units in the last place) is cheap. Masks are
// taken from each row's range of seen rows, in blocks that are seen in part. Short calls,
// bound by latency: 128 tokens, 4 heads of 64, 6.2 us; a step of 512 tokens, 8 heads of
// 128, three documents, cap and bias, 13 + 18 + 20 us (forward, dQ~, dV).

#include <algorithm>

#include "f32_tile.h"
#include "scored_device.h"
#include "tree_device.h"

namespace kl {
namespace {

constexpr int NW = 8;  // waves per workgroup

// A pair's score in log2 units; the shift by the row's maximum stays a separate term.
template <bool CAP, bool BIAS>
struct ExactForm {
  static constexpr bool kFalling = false;
  float scale, cap, scale2, cap2, inv;
  __device__ __forceinline__ ExactForm(float scale_, float cap_)
      : scale(scale_), cap(cap_), scale2(scale_ * kScoredLog2e), cap2(cap_ * kScoredLog2e),
        inv(CAP ? scale_ / cap_ : 0.f) {}
  __device__ __forceinline__ float A() const { return CAP || BIAS ? 1.f : scale2; }
  __device__ __forceinline__ float C() const { return 0.f; }
  static __device__ __forceinline__ float unseen() { return -INFINITY; }
  static __device__ __forceinline__ float best(float a, float b) { return fmaxf(a, b); }
  // tanh of the score over the cap.
  __device__ __forceinline__ float bent(float s) const { return tanhf(s * inv); }
  template <class Bias>
  __device__ __forceinline__ float with(float s, float t, Bias bias) const {
    float x = CAP ? t * cap2 : BIAS ? s * scale2 : s;
    if constexpr (BIAS) x = bias(x);
    return x;
  }
  template <class Bias>
  __device__ __forceinline__ float key(float s, Bias bias) const {
    return with(s, CAP ? bent(s) : 0.f, bias);
  }
  __device__ __forceinline__ float shifted(float k, float shift) const {
    return CAP || BIAS ? k + shift : fmaf(scale2, k, shift);
  }
};

// Values that are not finite in this lane's part of a staged block become zeros.
template <int D>
__device__ __forceinline__ void keep_finite(float* tile, int r, int g) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    f32x4_t* at = reinterpret_cast<f32x4_t*>(tile + r * Block<D>::PITCH + 16 * s + 4 * g);
    f32x4_t x = *at;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = not_finite(x[i]) ? 0.f : x[i];
    *at = x;
  }
}

// Merge of NW waves' (m, l, o) of the 16 own rows, in wave order: out(row, column, x, m,
// l) gets the sums relative to the common reference m.
template <int D, class Out>
__device__ __forceinline__ void merge_waves_f32(float* lds, float* tile, float (*s_ml)[16][2], int wave,
                                                int r, int g, float m, float l,
                                                const f32x4_t (&o)[D / 16], Out out) {
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    s_ml[wave][r][0] = m;
    s_ml[wave][r][1] = l;
  }
  __syncthreads();
  auto total = [&](int row, float& mx) {
    mx = s_ml[0][row][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) mx = fmaxf(mx, s_ml[w][row][0]);
    const float ms = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum = fmaf(s_ml[w][row][1], fast_exp2(s_ml[w][row][0] - ms), sum);
    return sum;
  };
  float mx;
  total(r, mx);
  const float f = fast_exp2(m - (mx == -INFINITY ? 0.f : mx));
  merge_sum<D, NW>(lds, tile, r, g, f, o, [&](int row, int c, f32x4_t x) {
    float mr;
    const float sum = total(row, mr);
    out(row, c, x, mr, sum);
  });
}

// One 16-row block of values against the own rows: weights, and the running sums.
template <int D, class Form, class Unseen, class Bias>
__device__ __forceinline__ void take_block(const Form& form, float* tile, int r, int g, f32x4_t s,
                                           f32x4_t (&o)[D / 16][1], float (&m)[1], float (&l)[1], bool edge,
                                           Unseen unseen, Bias bias) {
  f32x4_t sc[1][1] = {{s}};
  const bool bad = soften<D, 1, 1>(form, sc, o, m, l, edge, unseen, bias);
  if (bad) keep_finite<D>(tile, r, g);
  f32x4_t acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) acc[i] = o[i][0];
  add_weighted<D>(tile, r, g, sc[0][0], acc);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i][0] = acc[i];
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void forward_kernel(ScoredParams p) {
  constexpr int S = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds_f32[];
  __shared__ float s_ml[NW][16][2];
  const HeadTile ht(p, 16);
  const int h = ht.h, kg = ht.g, b = ht.b, q0 = ht.qt * 16;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const tile = lds_f32 + wave * Block<D>::FLOATS;
  const SeenRange seen = seen_range(p, b, min(q0 + r, p.N - 1));
  SeenBounds sb;
  sb.add(seen);
  sb.over_rows();
  sb.make_uniform();
  const bool any = sb.any_lo < sb.any_hi;
  const int t0 = any ? sb.any_lo / 16 : 0, nblk = any ? (sb.any_hi + 15) / 16 : 0;

  const long vs = (long)p.G * D, qs = (long)p.H * D;
  const float* V = static_cast<const float*>(p.v) + (size_t)b * p.N * vs + (size_t)kg * D;
  const float* Q = static_cast<const float*>(p.q) + (size_t)b * p.N * qs + (size_t)h * D;
  f32x4_t v[S], q[S], o[S][1];
  if (t0 + wave < nblk) load_rows<D>(V, vs, (t0 + wave) * 16 + r, p.N, g, v);
  load_rows<D>(Q, qs, q0 + r, p.N, g, q);
  const ExactForm<CAP, BIAS> form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  float m[1] = {-INFINITY}, l[1] = {0.f};
#pragma unroll
  for (int s = 0; s < S; ++s) o[s][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int t = t0 + wave; t < nblk; t += NW) {
    const int j0 = t * 16;
    stage_rows<D>(tile, r, g, v);
    const f32x4_t sc = dot_rows<D>(v, q, f32x4_t{0.f, 0.f, 0.f, 0.f});
    if (t + NW < nblk) load_rows<D>(V, vs, j0 + NW * 16 + r, p.N, g, v);
    const bool edge = j0 < sb.all_lo || j0 + 16 > sb.all_hi;
    take_block<D>(
        form, tile, r, g, sc, o, m, l, edge,
        [&](int, int, int i) { return (j0 + 4 * g + i < seen.lo) | (j0 + 4 * g + i >= seen.hi); },
        [&](float x, int, int, int i) { return fmaf(-slope, fabsf((float)(q0 + r - j0 - 4 * g - i)), x); });
  }
  f32x4_t acc[S];
#pragma unroll
  for (int s = 0; s < S; ++s) acc[s] = o[s][0];
  merge_waves_f32<D>(lds_f32, tile, s_ml, wave, r, g, m[0], l[0], acc,
                     [&](int row, int c, f32x4_t x, float mr, float sum) {
    if (q0 + row >= p.N) return;
    const size_t at = (((size_t)b * p.N + q0 + row) * p.H + h) * D + c;
    const f32x4_t y = x * (sum == 0.f ? 0.f : 1.f / sum);
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = y;
    if (p.out_f32) *reinterpret_cast<f32x4_t*>(p.out_f32 + at) = y;
    if (p.lse && c == 0)
      p.lse[((size_t)b * p.H + h) * p.N + q0 + row] =
          sum == 0.f ? -INFINITY : (mr + __log2f(sum)) * kScoredLn2;
  });
}

// Publishes for dV, from the first head's workgroups, what each query row and each
// 16-row block sees, and Dd.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void dq_kernel(ScoredParams p) {
  constexpr int S = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds_f32[];
  const HeadTile ht(p, 16);
  const int h = ht.h, kg = ht.g, b = ht.b, q0 = ht.qt * 16;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const tile = lds_f32 + wave * Block<D>::FLOATS;
  const SeenRange seen = seen_range(p, b, min(q0 + r, p.N - 1));
  SeenBounds sb, pub;
  sb.add(seen);
  pub.add(q0 + r < p.N ? seen : SeenRange{0, 0});
  sb.over_rows();
  pub.over_rows();
  sb.make_uniform();
  if (h == 0 && threadIdx.x < 16) {
    if (q0 + r < p.N) {
      p.row_lo[(size_t)b * p.N + q0 + r] = seen.lo;
      p.row_hi[(size_t)b * p.N + q0 + r] = seen.hi;
    }
    if (r == 0)
      static_cast<i32x4*>(p.tile_sees)[(size_t)b * ((p.N + 15) / 16) + ht.qt] =
          i32x4{pub.any_lo, pub.any_hi, pub.all_lo, pub.all_hi};
  }
  const bool any = sb.any_lo < sb.any_hi;
  const int t0 = any ? sb.any_lo / 16 : 0, nblk = any ? (sb.any_hi + 15) / 16 : 0;

  const long vs = (long)p.G * D, qs = (long)p.H * D;
  const float* V = static_cast<const float*>(p.v) + (size_t)b * p.N * vs + (size_t)kg * D;
  const size_t head = (size_t)b * p.N * qs + (size_t)h * D;
  f32x4_t v[S], q[S], go[S], o[S], acc[S];
  if (t0 + wave < nblk) load_rows<D>(V, vs, (t0 + wave) * 16 + r, p.N, g, v);
  load_rows<D>(static_cast<const float*>(p.q) + head, qs, q0 + r, p.N, g, q);
  load_rows<D>(static_cast<const float*>(p.dout) + head, qs, q0 + r, p.N, g, go);
  load_rows<D>((p.out_f32 ? p.out_f32 : static_cast<const float*>(p.out_in)) + head, qs, q0 + r, p.N, g, o);
  const size_t row = ((size_t)b * p.H + h) * p.N + min(q0 + r, p.N - 1);
  const float shift = -p.lse[row] * kScoredLog2e;
  float dd = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      dd = fmaf(o[s][j], go[s][j], dd);
      acc[s][j] = 0.f;
    }
  dd += __shfl_xor(dd, 16);
  dd += __shfl_xor(dd, 32);
  if (wave == 0 && g == 0 && q0 + r < p.N) p.Dd[row] = dd;
  const ExactForm<CAP, BIAS> form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  for (int t = t0 + wave; t < nblk; t += NW) {
    const int j0 = t * 16;
    stage_rows<D>(tile, r, g, v);
    const f32x4_t sc = dot_rows<D>(v, q, f32x4_t{0.f, 0.f, 0.f, 0.f});
    const f32x4_t dp = dot_rows<D>(v, go, f32x4_t{0.f, 0.f, 0.f, 0.f});
    if (t + NW < nblk) load_rows<D>(V, vs, j0 + NW * 16 + r, p.N, g, v);
    const bool edge = j0 < sb.all_lo || j0 + 16 > sb.all_hi;
    f32x4_t dz;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + 4 * g + i;
      const bool unseen = (j < seen.lo) | (j >= seen.hi);
      const bool odd = not_finite(sc[i]) | not_finite(dp[i]);
      const float t1 = CAP ? form.bent(sc[i]) : 0.f;
      const float x = form.with(sc[i], t1, [&](float y) { return fmaf(-slope, fabsf((float)(q0 + r - j)), y); });
      float z = fast_exp2(form.shifted(x, shift)) * (dp[i] - dd);
      if constexpr (CAP) z *= fmaf(-t1, t1, 1.f);
      bad |= unseen & odd;
      z = odd ? __builtin_nanf("") : z;
      dz[i] = unseen ? 0.f : z;
    }
    if (edge && __builtin_amdgcn_ballot_w64(bad)) keep_finite<D>(tile, r, g);
    add_weighted<D>(tile, r, g, dz, acc);
  }
  float* out = static_cast<float*>(p.dq);
  merge_sum<D, NW>(lds_f32, tile, r, g, p.scale, acc, [&](int rr, int c, f32x4_t x) {
    if (q0 + rr < p.N) *reinterpret_cast<f32x4_t*>(out + head + (size_t)(q0 + rr) * qs + c) = x;
  });
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void dv_kernel(ScoredParams p) {
  constexpr int S = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds_f32[];
  __shared__ int s_first[NW], s_last[NW];
  const int R = p.H / p.G, kg = blockIdx.x % p.G, rest = blockIdx.x / p.G;
  const int b = rest % p.B, kv0 = rest / p.B * 16;  // under the causal mask the first blocks are the heaviest
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const tq = lds_f32 + wave * 2 * Block<D>::FLOATS;
  float* const tg = tq + Block<D>::FLOATS;

  // The query blocks from the first to the last that sees one of these rows.
  const int blocks = (p.N + 15) / 16;
  const i32x4* sees = static_cast<const i32x4*>(p.tile_sees) + (size_t)b * blocks;
  int first = blocks, last = 0;
  for (int t = threadIdx.x; t < blocks; t += NW * 64) {
    const i32x4 s = sees[t];
    if ((s.x < kv0 + 16) & (s.y > kv0)) {
      first = min(first, t);
      last = max(last, t + 1);
    }
  }
  first = wave_reduce(first, [](int x, int y) { return min(x, y); });
  last = wave_reduce(last, [](int x, int y) { return max(x, y); });
  if (lane == 0) {
    s_first[wave] = first;
    s_last[wave] = last;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    first = min(first, s_first[w]);
    last = max(last, s_last[w]);
  }
  first = __builtin_amdgcn_readfirstlane(first);
  last = __builtin_amdgcn_readfirstlane(last);
  const int per = max(last - first, 0), items = R * per;
  typedef const __attribute__((address_space(4))) i32x4 const_i32x4;
  // The wave's items are every NW-th (head, query block); those that see nothing of the
  // block are passed over.
  auto seek = [&](int it) {
    for (; it < items; it += NW) {
      const i32x4 s = ((const_i32x4*)sees)[first + it % per];
      if (s.x < kv0 + 16 && s.y > kv0) break;
    }
    return it;
  };

  const long qs = (long)p.H * D;
  const float* Q = static_cast<const float*>(p.q) + (size_t)b * p.N * qs;
  const float* dO = static_cast<const float*>(p.dout) + (size_t)b * p.N * qs;
  f32x4_t v[S], q[S], go[S], acc[S];
  float lse[4], dd[4];
  int lo[4], hi[4];
  auto load = [&](int it) {
    const int h = kg * R + it / per, q0 = (first + it % per) * 16;
    load_rows<D>(Q + (size_t)h * D, qs, q0 + r, p.N, g, q);
    load_rows<D>(dO + (size_t)h * D, qs, q0 + r, p.N, g, go);
    const size_t row = ((size_t)b * p.H + h) * p.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int qq = q0 + 4 * g + i, qc = min(qq, p.N - 1);
      lse[i] = p.lse[row + qc];
      dd[i] = p.Dd[row + qc];
      lo[i] = p.row_lo[(size_t)b * p.N + qc];
      hi[i] = qq < p.N ? p.row_hi[(size_t)b * p.N + qc] : 0;  // rows past the end see nothing
    }
  };
  int it = seek(wave);
  if (it < items) load(it);
  load_rows<D>(static_cast<const float*>(p.v) + (size_t)b * p.N * p.G * D + (size_t)kg * D, (long)p.G * D,
               kv0 + r, p.N, g, v);
#pragma unroll
  for (int s = 0; s < S; ++s) acc[s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const ExactForm<CAP, BIAS> form(p.scale, p.cap);
  while (it < items) {
    const int q0 = (first + it % per) * 16, h = kg * R + it / per, next = seek(it + NW);
    const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
    stage_rows<D>(tq, r, g, q);
    stage_rows<D>(tg, r, g, go);
    const f32x4_t sc = dot_rows<D>(q, v, f32x4_t{0.f, 0.f, 0.f, 0.f});
    const f32x4_t dp = dot_rows<D>(go, v, f32x4_t{0.f, 0.f, 0.f, 0.f});
    f32x4_t w, dz;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int kv = kv0 + r;
      const bool unseen = (kv < lo[i]) | (kv >= hi[i]);
      const bool odd = not_finite(sc[i]) | not_finite(dp[i]);
      const float t1 = CAP ? form.bent(sc[i]) : 0.f;
      const float x = form.with(
          sc[i], t1, [&](float y) { return fmaf(-slope, fabsf((float)(q0 + 4 * g + i - kv)), y); });
      float pw = fast_exp2(form.shifted(x, -lse[i] * kScoredLog2e));
      float z = pw * (dp[i] - dd[i]) * p.scale;
      if constexpr (CAP) z *= fmaf(-t1, t1, 1.f);
      bad |= unseen & odd;
      pw = odd ? __builtin_nanf("") : pw;
      z = odd ? __builtin_nanf("") : z;
      w[i] = unseen ? 0.f : pw;
      dz[i] = unseen ? 0.f : z;
    }
    if (next < items) load(next);
    if (__builtin_amdgcn_ballot_w64(bad)) {
      keep_finite<D>(tq, r, g);
      keep_finite<D>(tg, r, g);
    }
    add_weighted<D>(tg, r, g, w, acc);
    add_weighted<D>(tq, r, g, dz, acc);
    it = next;
  }
  __syncthreads();
  float* out = static_cast<float*>(p.dv);
  merge_sum<D, NW>(lds_f32, lds_f32 + wave * Block<D>::FLOATS, r, g, 1.f, acc, [&](int rr, int c, f32x4_t x) {
    if (kv0 + rr < p.N)
      *reinterpret_cast<f32x4_t*>(out + (((size_t)b * p.N + kv0 + rr) * p.G + kg) * D + c) = x;
  });
}

// Drafted tokens: 16 query rows (token, head of the group) against one chunk of a
// sequence's rows, whose 16-row blocks the waves share; a block lies in one page.
template <int D, bool CAP, bool BIAS, bool PAGED>
__global__ __launch_bounds__(NW * 64, 2) void tree_kernel(TreeParams p) {
  constexpr int S = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds_f32[];
  __shared__ float s_ml[NW][16][2];
  __shared__ int s_depth[BIAS ? kMaxDrafts : 1];
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R = p.H / p.G, M = p.T * R, blocks = (M + 15) / 16;
  const int kg = blockIdx.x % p.G, m0 = (int)(blockIdx.x / p.G % blocks) * 16;
  const int c = blockIdx.x / p.G / blocks;
  float* const tile = lds_f32 + wave * Block<D>::FLOATS;
  const ExactForm<CAP, BIAS> form(p.scale, p.cap);
  TreeWalk walk(p, lane, c);
  TreeSeg sp;
  while (walk.next(p, lane, sp)) {
    const int row0 = sp.tile0 * kTreeTile;
    const int nblk = (min(sp.rows - row0, sp.tiles * kTreeTile) + 15) / 16;
    const float* data = static_cast<const float*>(p.data);
    // The rows of block t, of which `n` exist; none outside the cache.
    auto rows_of = [&](int t, int& n) {
      const int j = row0 + t * 16;
      n = min(sp.rows - j, 16);
      if constexpr (PAGED) {
        const int blk =
            ((const __attribute__((address_space(4))) int*)p.table)[(size_t)sp.b * p.max_blocks + (j >> p.block_shift)];
        const bool ok = blk >= 0 && blk < p.num_blocks;
        if (!ok) n = 0;
        return data + ((((size_t)(ok ? blk : 0) * p.G + kg) << p.block_shift) + (j & ((1 << p.block_shift) - 1))) * D;
      } else {
        return data + (((size_t)sp.b * p.G + kg) * p.L_max + j) * D;
      }
    };
    f32x4_t v[S], q[S], o[S][1];
    int live = 0, live_next = 0;
    if (wave < nblk) {
      const float* V = rows_of(wave, live_next);
      load_rows<D>(V, D, r, live_next, g, v);
    }
    const int mr = min(m0 + r, M - 1), tok = mr / R;
    load_rows<D>(static_cast<const float*>(p.q) + (((size_t)sp.b * p.T + tok) * p.H + kg * R + mr % R) * D, D, 0, 1,
                 g, q);
    const uint64_t word = tree_word(p, sp.b, tok);
    const int place = tree_depth(word, tok);
    float slope = 0.f;
    if constexpr (BIAS) {
      slope = p.slopes[kg * R + mr % R] * kScoredLog2e;
      for (int t = threadIdx.x; t < p.T; t += NW * 64) s_depth[t] = tree_depth(tree_word(p, sp.b, t), t);
      __syncthreads();
    }
    float m[1] = {-INFINITY}, l[1] = {0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) o[s][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int t = wave; t < nblk; t += NW) {
      const int j0 = row0 + t * 16;
      live = live_next;
      stage_rows<D>(tile, r, g, v);
      const f32x4_t sc = dot_rows<D>(v, q, f32x4_t{0.f, 0.f, 0.f, 0.f});
      if (t + NW < nblk) {
        const float* V = rows_of(t + NW, live_next);
        load_rows<D>(V, D, r, live_next, g, v);
      }
      const bool edge = j0 + 16 > sp.n || live < 16;
      const int jl = j0 + 4 * g;
      take_block<D>(
          form, tile, r, g, sc, o, m, l, edge,
          [&](int, int, int i) {
            const int u = jl + i - sp.n;
            return (4 * g + i >= live) | ((u >= 0) & ((word >> (u & 63) & 1) == 0));
          },
          [&](float x, int, int, int i) {
            const int j = jl + i;
            int d = sp.n + place - j;
            if (BIAS && edge && j >= sp.n) d = abs(place - s_depth[min(j - sp.n, p.T - 1)]);
            return fmaf(-slope, (float)d, x);
          });
    }
    f32x4_t acc[S];
#pragma unroll
    for (int s = 0; s < S; ++s) acc[s] = o[s][0];
    merge_waves_f32<D>(lds_f32, tile, s_ml, wave, r, g, m[0], l[0], acc,
                       [&](int row, int col, f32x4_t x, float mx, float sum) {
      const int m1 = m0 + row;
      if (m1 >= M) return;
      if (sp.whole) {
        float* dst = static_cast<float*>(p.out) + (((size_t)sp.b * p.T + m1 / R) * p.H + kg * R + m1 % R) * D + col;
        *reinterpret_cast<f32x4_t*>(dst) = x * (sum == 0.f ? 0.f : 1.f / sum);
      } else {
        *reinterpret_cast<f32x4_t*>(tree_part(p, sp.slot, kg, m1) + col) = x;
        if (col == 0) {
          float* ml = tree_part_ml(p, sp.slot, kg, m1);
          ml[0] = mx;
          ml[1] = sum;
        }
      }
    });
    __syncthreads();  // the results have been read: the next segment may fill their place
  }
}

template <class K, class P>
hipError_t launch(K kern, const P& p, unsigned grid, int lds, std::atomic<uint32_t>& done, hipStream_t st) {
  const hipError_t e = set_max_lds(reinterpret_cast<const void*>(kern), lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(NW * 64), lds, st, p);
  return hipGetLastError();
}

// f(cap, bias) with the template arguments of a call.
template <class P, class F>
hipError_t pick_form(const P& p, F f) {
  using Y = std::true_type;
  using N = std::false_type;
  if (p.cap > 0.f) return p.slopes ? f(Y{}, Y{}) : f(Y{}, N{});
  return p.slopes ? f(N{}, Y{}) : f(N{}, N{});
}

template <int D>
hipError_t forward(const ScoredParams& p, hipStream_t st) {
  return pick_form(p, [&](auto cap, auto bias) {
    static std::atomic<uint32_t> done{0};
    return launch(forward_kernel<D, decltype(cap)::value, decltype(bias)::value>, p,
                  (unsigned)p.H * p.B * ((p.N + 15) / 16), NW * Block<D>::FLOATS * 4, done, st);
  });
}

template <int D>
hipError_t backward(const ScoredParams& p, hipStream_t st) {
  return pick_form(p, [&](auto cap, auto bias) {
    static std::atomic<uint32_t> done_q{0}, done_v{0};
    const unsigned blocks = (unsigned)p.B * ((p.N + 15) / 16);
    const hipError_t e = launch(dq_kernel<D, decltype(cap)::value, decltype(bias)::value>, p, p.H * blocks,
                                NW * Block<D>::FLOATS * 4, done_q, st);
    if (e != hipSuccess) return e;
    return launch(dv_kernel<D, decltype(cap)::value, decltype(bias)::value>, p, p.G * blocks,
                  2 * NW * Block<D>::FLOATS * 4, done_v, st);
  });
}

template <int D>
hipError_t tree(const TreeParams& p, hipStream_t st) {
  const hipError_t e = pick_form(p, [&](auto cap, auto bias) {
    static std::atomic<uint32_t> done_p{0}, done_c{0};
    constexpr bool C = decltype(cap)::value, A = decltype(bias)::value;
    const unsigned grid = (unsigned)p.chunks * (p.per > 0 ? p.B : 1) * ((p.T * (p.H / p.G) + 15) / 16) * p.G;
    const int lds = NW * Block<D>::FLOATS * 4;
    return p.paged ? launch(tree_kernel<D, C, A, true>, p, grid, lds, done_p, st)
                   : launch(tree_kernel<D, C, A, false>, p, grid, lds, done_c, st);
  });
  return e != hipSuccess || !p.part ? e : launch_tree_merge(p, st);
}

}  // namespace

hipError_t launch_scored_forward_f32(const ScoredParams& p, hipStream_t st) {
  return p.D == 128 ? forward<128>(p, st) : forward<64>(p, st);
}

hipError_t launch_scored_backward_f32(const ScoredParams& p, hipStream_t st) {
  return p.D == 128 ? backward<128>(p, st) : backward<64>(p, st);
}

hipError_t launch_tree_decode_f32(const TreeParams& p, hipStream_t st) {
  return p.D == 128 ? tree<128>(p, st) : tree<64>(p, st);
}

}  // namespace kl
