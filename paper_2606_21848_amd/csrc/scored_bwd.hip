// Scored keyless attention, bf16 backward on the matrix cores. Per batch and head, with
// x the capped and biased score and z the plain one:
//   P   = exp(x - lse),  dP = dO V^T,  Dd = rowsum(dO * O)
//   dx  = P * (dP - Dd),  dz = dx (1 - tanh^2(z / cap))
//   dQ~ = scale dz V
//   dV  = P^T dO + scale dz^T Q~   (both roles of the values, every head of the group)
//
// scored_dq_kernel (one workgroup per 128 query rows and head; value tiles stream
// through LDS, queries and dO stay in registers) publishes for the second kernel what
// each query row and each 32-row query block sees, and Dd. scored_dv_kernel (one
// workgroup per 192 value rows and group; tiles of Q~ and dO stream through LDS, the
// values stay in registers) walks the query tiles that see any of its rows, for every
// head of its group, and masks only in tiles that see them in part. No atomics.
// Scores come out with one query per lane in the first kernel and one value row per
// lane in the second, so that in both the weights are the next product's second operand
// as they stand. Queries and weights are not multiplied by the scale before a rounding; P
// and dz are rounded to bf16 once each, as operands of the last products.
//
// 8192 tokens in two documents, 32 heads on 8 groups of 128, cap 50: 1.42 ms with the sum
// of the splits. Bound by instruction issue as the forward is (the dV kernel: matrix
// instructions 28% of the cycles, vector ones 30%, waits for LDS and barriers 33% at two
// waves per SIMD, all 256 registers in use).

#include <algorithm>
#include <type_traits>

#include "attn_tile.h"
#include "scored_device.h"

namespace kl {
namespace {

constexpr int kThreads = 256;
constexpr int kTileRows = 64;
constexpr int kStages = 3;           // value tiles in LDS (dQ~)
constexpr int QB = 2, BQ = 64 * QB;  // 16-row query blocks per wave, query rows per workgroup (dQ~)
// Fewest (head, query tile) pairs of a split of the dV sums (2 packed sequences of 1000
// tokens, 12 heads, a training step: 83 us; 86 with 1, 90 with 3, 103 with 4).
constexpr int kLeastItems = 2;
constexpr int KVB = 3, BKV = 64 * KVB;  // value blocks per wave, value rows per workgroup (dV)

// One 4-byte-per-lane copy from global memory straight into LDS.
__device__ __forceinline__ void copy_dword_to_lds(const void* gbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(voff), "s"(gbase), "s"(lds)
               : "memory", "m0");
}

// The lane's number, computed anew at each call: what is derived from it is then not kept
// in registers from one loop iteration to the next.
__device__ __forceinline__ int lane_again() {
  unsigned all = ~0u;
  asm volatile("" : "+s"(all));
  return (int)__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
}

// P of one pair from its dot product, and `scale` times the slope of the cap there (dz is
// the product of both with dP - Dd). shift = C - lse in log2 units.
template <class Form, bool CAP, bool BIAS>
__device__ __forceinline__ void weigh(const Form& form, float s, float slope, float dist, float shift, float scale,
                                      float& w, float& bend) {
  if constexpr (CAP) {
    const float k = form.bent(s);
    float x = k;
    if constexpr (BIAS) x = fmaf(-slope, fabsf(dist), fmaf(k, -2.f * form.cap2, form.cap2));
    w = fast_exp2(form.shifted(x, shift));
    const float k4 = k * (4.f * scale);
    bend = fmaf(-k4, k, k4);  // 1 - tanh^2 = 4 k (1 - k)
  } else {
    w = fast_exp2(form.shifted(form.key(s, [&](float x) { return fmaf(-slope, fabsf(dist), x); }), shift));
    bend = scale;
  }
}

// What the 32 query rows from q0 on see (lane: rows q0 + 16 qb + fr), into `seen` and the
// bounds returned; `publish`: for the dV kernel too (rows past the end see nothing there, so
// that a block with a tail counts as seen in part).
__device__ __forceinline__ SeenBounds seen_by_rows(const ScoredParams& p, int b, int q0, int fr, int grp,
                                                   bool publish, SeenRange (&seen)[QB]) {
  SeenBounds sb, pub;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int q = q0 + qb * 16 + fr;
    seen[qb] = seen_range(p, b, min(q, p.N - 1));
    sb.add(seen[qb]);
    pub.add(q < p.N ? seen[qb] : SeenRange{0, 0});
    if (publish && grp == 0 && q < p.N) {
      p.row_lo[(size_t)b * p.N + q] = seen[qb].lo;
      p.row_hi[(size_t)b * p.N + q] = seen[qb].hi;
    }
  }
  sb.over_rows();
  sb.make_uniform();
  if (publish && q0 < p.N) {
    pub.over_rows();
    if (fr == 0 && grp == 0)
      static_cast<i32x4*>(p.tile_sees)[(size_t)b * ((p.N + 31) / 32) + q0 / 32] =
          i32x4{pub.any_lo, pub.any_hi, pub.all_lo, pub.all_hi};
  }
  return sb;
}

// Over a query's four lanes.
__device__ __forceinline__ float over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Query row q0 + 16 qb + fr, columns 32 ks + 8 grp .. + 7, of Q~ and dO, what dP starts
// from (-Dd), and the shift of its scores. Dd comes from the forward's output; correct()
// makes up for its rounding.
template <int D, class Form>
__device__ __forceinline__ void load_query_rows(const ScoredParams& p, const Form& form, int b, int h, int q0,
                                                int fr, int grp, bf16x8_t (&qf)[QB][D / 32],
                                                bf16x8_t (&df)[QB][D / 32], f32x4_t (&ndd)[QB],
                                                float (&shift)[QB]) {
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int qq = min(q0 + qb * 16 + fr, p.N - 1);
    const size_t at = (((size_t)b * p.N + qq) * p.H + h) * D + grp * 8;
    const size_t row = ((size_t)b * p.H + h) * p.N + qq;
    float d0 = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      qf[qb][ks] = __builtin_bit_cast(
          bf16x8_t, *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + at + ks * 32));
      const u32x4 gw = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.dout) + at + ks * 32);
      df[qb][ks] = __builtin_bit_cast(bf16x8_t, gw);
      const u32x4 o = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.out_in) + at + ks * 32);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        d0 = fmaf(bf16_lo(gw[j]), bf16_lo(o[j]), fmaf(bf16_hi(gw[j]), bf16_hi(o[j]), d0));
    }
    d0 = over_groups(d0);
    ndd[qb] = f32x4_t{-d0, -d0, -d0, -d0};
    shift[qb] = form.C() - p.lse[row] * kScoredLog2e;
  }
}

// dQ~^T += V^T dz^T for the 32 value rows from j0 on, staged at `fi` (relative rows at
// `rows`): S^T = V Q~^T and dP^T = V dO^T share each value-row fragment read, and dz^T is
// the last product's second operand. off and bent gather sum P (dP - Dd) and, under a cap,
// sum P bend over the lane's rows: see correct().
template <int D, bool CAP, bool BIAS, int ROW, class Form>
__device__ __forceinline__ void dq_step(const Form& form, const FragOffsets<D>& fi, int rows, int j0, int q0,
                                        int fr, int grp, bool edge, float slope, const SeenRange (&seen)[QB],
                                        const bf16x8_t (&qf)[QB][D / 32], const bf16x8_t (&df)[QB][D / 32],
                                        const f32x4_t (&ndd)[QB], const float (&shift)[QB],
                                        f32x4_t (&acc)[D / 16][QB], float (&off)[QB], float (&bent)[QB]) {
  constexpr int KS = D / 32, DB = D / 16;
        f32x4_t sc[2][QB], dp[2][QB];
        bf16x8_t va[2][KS];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int kd = 0; kd < KS; ++kd) va[hh][kd] = lds_rows(fi.s(kd) + rows + hh * 16 * ROW);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int kd = 0; kd < KS; ++kd)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
              sc[hh][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  va[hh][kd], qf[qb][kd], kd == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[hh][qb], 0, 0, 0);
              dp[hh][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[hh][kd], df[qb][kd],
                                                                   kd == 0 ? ndd[qb] : dp[hh][qb], 0, 0, 0);
            }
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, KS, 0);
#pragma unroll
        for (int kd = 0; kd < KS; ++kd) {
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2 * QB, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2 * QB * KS, 0);
        // Lane: rows jl + 16 hh + r of query q0 + 16 qb + fr.
        const int jl = j0 + grp * 4;
        auto unseen = [&](int qb, int hh, int r) {
          const int j = jl + hh * 16 + r;
          return (j < seen[qb].lo) | (j >= seen[qb].hi);
        };
        bool bad = false;  // see the forward: values that a query must not see are not finite
        if (edge) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                bad |= unseen(qb, hh, r) & (not_finite(sc[hh][qb][r]) | not_finite(dp[hh][qb][r]));
          bad = __builtin_amdgcn_ballot_w64(bad) != 0;
          if (bad) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  dp[hh][qb][r] = not_finite(sc[hh][qb][r]) ? __builtin_nanf("") : dp[hh][qb][r];
          }
        }
        bf16x8_t pf[QB];
        auto weights = [&](auto masked) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            const float dist = (float)(q0 + qb * 16 + fr - jl);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float w, bend;
                weigh<Form, CAP, BIAS>(form, sc[hh][qb][r], slope, dist - (float)(hh * 16 + r), shift[qb], 1.f, w,
                                       bend);
                float wd = w * dp[hh][qb][r];
                if constexpr (decltype(masked)::value) {
                  const bool no = unseen(qb, hh, r);
                  w = no ? 0.f : w;
                  wd = no ? 0.f : wd;
                  bend = no ? 0.f : bend;
                }
                off[qb] += wd;
                if constexpr (CAP) bent[qb] = fmaf(w, bend, bent[qb]);
                sc[hh][qb][r] = CAP ? wd * bend : wd;
              }
          }
        };
        if (edge) weights(std::true_type{});
        else weights(std::false_type{});
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) pf[qb] = pack8(sc[0][qb], sc[1][qb]);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          bf16x8_t a = lds_columns<ROW>(fi.t(db) + rows);
          if (bad) a = finite_or_zero(a);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            acc[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[qb], acc[db][qb], 0, 0, 0);
        }
}

// Dd from the forward's output carries the bf16 roundings of that output and of its
// weights, the same for a whole row: off = sum P (dP - Dd) is what it lacks, and
// sum P bend V off, taken as (sum P bend) O off (without a cap just that), what dQ~ has too
// much. Error of dQ~ against 64 bits (8192 tokens, two documents, cap 50): 0.0023, of which
// the roundings of dz and of the result are 0.0016 each; 0.0025 with the fp32 output and no
// correction, for 80 us more in 1500.
__device__ __forceinline__ f32x4_t correct(f32x4_t dq, u32x2 out, float f) {
  return f32x4_t{fmaf(-f, bf16_lo(out[0]), dq[0]), fmaf(-f, bf16_hi(out[0]), dq[1]),
                 fmaf(-f, bf16_lo(out[1]), dq[2]), fmaf(-f, bf16_hi(out[1]), dq[3])};
}
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void scored_dq_kernel(ScoredParams p) {
  using T = AttnTile<D, kTileRows>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int KS = D / 32, DB = D / 16;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ int s_sees[4][2];
  const HeadTile ht(p, BQ);
  const int h = ht.h, g = ht.g, b = ht.b, qt = ht.qt;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  const int q0 = qt * BQ + wave * 16 * QB;

  SeenRange seen[QB];
  SeenBounds sb = seen_by_rows(p, b, q0, fr, grp, h == 0, seen);
  if (q0 >= p.N) sb.any_lo = sb.any_hi = 0;
  if (lane == 0) {
    s_sees[wave][0] = sb.any_hi > sb.any_lo ? sb.any_lo : 0x7fffffff;
    s_sees[wave][1] = sb.any_hi;
  }
  __syncthreads();
  int lo = s_sees[0][0], hi = s_sees[0][1];
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    lo = min(lo, s_sees[w][0]);
    hi = max(hi, s_sees[w][1]);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const int t0 = lo < hi ? lo / kTileRows : 0;
  const int ntiles = lo < hi ? (hi + kTileRows - 1) / kTileRows - t0 : 0;

  const size_t row_bytes = (size_t)p.G * D * 2;
  const unsigned char* gV = static_cast<const unsigned char*>(p.v) + ((size_t)b * p.N * p.G + g) * D * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  const TileCopy<D> cp(wave, lane, row_bytes);
  auto issue = [&](int t, int stage) {
    cp.issue(gV, row_bytes, (t0 + t) * kTileRows, p.N, wave, lane, lds0 + stage * T::BYTES);
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    if (s < ntiles) issue(s, s);

  const Form form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  bf16x8_t qf[QB][KS], df[QB][KS];
  f32x4_t ndd[QB], acc[DB][QB];
  float shift[QB];
  load_query_rows<D>(p, form, b, h, q0, fr, grp, qf, df, ndd, shift);
  float off[QB] = {}, bent[QB] = {};
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const FragOffsets<D> fo(fr, grp);
  KL_WAIT_VMCNT(0);
  int stage = 0;
  for (int t = 0; t < ntiles; ++t) {
    if (t + 1 < ntiles) KL_WAIT_VMCNT((kStages - 2) * T::COPIES);
    else KL_WAIT_VMCNT(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage refilled below has been read
    __syncthreads();
    if (t + kStages - 1 < ntiles) issue(t + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
    const int j0 = (t0 + t) * kTileRows;
    const FragOffsets<D> fi = fo.at(lds0 + stage * T::BYTES);
    stage = stage == kStages - 1 ? 0 : stage + 1;
    if (j0 >= sb.any_hi || j0 + kTileRows <= sb.any_lo) continue;
    const bool edge = j0 < sb.all_lo || j0 + kTileRows > sb.all_hi;
    // One 32-row step at a time, which keeps half of the tile's scores live.
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      dq_step<D, CAP, BIAS, T::ROW>(form, fi, ks * 32 * T::ROW, j0 + 32 * ks, q0, fr, grp, edge, slope, seen, qf,
                                    df, ndd, shift, acc, off, bent);
  }
  // Lane holds dQ~^T[16 db + 4 grp + r][q].
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float lacks = over_groups(off[qb]), share = CAP ? over_groups(bent[qb]) : 1.f;
    const int q = q0 + qb * 16 + fr;
    if (q >= p.N) continue;
    if (grp == 0) p.Dd[((size_t)b * p.H + h) * p.N + q] = lacks - ndd[qb][0];
    const size_t at = (((size_t)b * p.N + q) * p.H + h) * D + grp * 4;
    const uint16_t* out = static_cast<const uint16_t*>(p.out_in) + at;
    uint16_t* dst = static_cast<uint16_t*>(p.dq) + at;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const f32x4_t x =
          correct(acc[db][qb], *reinterpret_cast<const u32x2*>(out + db * 16), lacks * share) * p.scale;
      *reinterpret_cast<u32x2*>(dst + db * 16) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    }
  }
}

// dQ~ for few query tiles: 32 query rows of one head per workgroup, its four waves sharing
// the 32-row value tiles through private two-stage rings; their sums are added once, in wave order.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void scored_dq_split_kernel(ScoredParams p) {
  constexpr int NW = 4, RV = 32, KS = D / 32, DB = D / 16;
  using T = AttnTile<D, RV>;
  using Copier = WaveCopier<D, RV>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int RING = 2 * T::BYTES;
  static_assert(RING == 32 * D * 4, "a wave's results fit its ring");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ float s_off[NW][32], s_bent[NW][32];
  const HeadTile ht(p, 32);
  const int h = ht.h, g = ht.g, b = ht.b, q0 = ht.qt * 32;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  SeenRange seen[QB];
  const SeenBounds sb = seen_by_rows(p, b, q0, fr, grp, h == 0 && wave == 0, seen);
  const bool any = sb.any_lo < sb.any_hi;
  const int t0 = any ? sb.any_lo / RV : 0, tend = any ? (sb.any_hi + RV - 1) / RV : 0;
  const size_t row_bytes = (size_t)p.G * D * 2;
  const unsigned char* gV = static_cast<const unsigned char*>(p.v) + ((size_t)b * p.N * p.G + g) * D * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  const uint32_t ring = lds0 + wave * RING;
  const Copier cp(lane, row_bytes);
  if (t0 + wave < tend) cp.issue(gV, row_bytes, (t0 + wave) * RV, p.N, lane, ring);
  const Form form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  bf16x8_t qf[QB][KS], df[QB][KS];
  f32x4_t ndd[QB], acc[DB][QB];
  float shift[QB];
  load_query_rows<D>(p, form, b, h, q0, fr, grp, qf, df, ndd, shift);
  float off[QB] = {}, bent[QB] = {};
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const FragOffsets<D> fo(fr, grp);
  int stage = 0;
  for (int t = t0 + wave; t < tend; t += NW) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other stage has been read
    if (t + NW < tend) {
      cp.issue(gV, row_bytes, (t + NW) * RV, p.N, lane, ring + (stage ^ 1) * T::BYTES);
      KL_WAIT_VMCNT(Copier::COPIES);
    } else {
      KL_WAIT_VMCNT(0);
    }
    asm volatile("" ::: "memory");
    const FragOffsets<D> fi = fo.at(ring + stage * T::BYTES);
    stage ^= 1;
    const int j0 = t * RV;
    dq_step<D, CAP, BIAS, T::ROW>(form, fi, 0, j0, q0, fr, grp, j0 < sb.all_lo || j0 + RV > sb.all_hi, slope, seen,
                                  qf, df, ndd, shift, acc, off, bent);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float lacks = over_groups(off[qb]), share = over_groups(bent[qb]);
    if (grp == 0) {
      s_off[wave][qb * 16 + fr] = lacks;
      s_bent[wave][qb * 16 + fr] = share;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) WaveSums<D>::put(ring, qb * 16 + fr, 4 * db + grp, acc[db][qb]);
  }
  __syncthreads();
  auto sum = [](const float (&x)[NW][32], int row) { return ((x[0][row] + x[1][row]) + x[2][row]) + x[3][row]; };
  if (wave == 0 && grp == 0) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int row = qb * 16 + fr;
      if (q0 + row < p.N) p.Dd[((size_t)b * p.H + h) * p.N + q0 + row] = sum(s_off, row) - ndd[qb][0];
    }
  }
  for (int e = threadIdx.x; e < 32 * D / 4; e += kThreads) {
    const int row = e / (D / 4), piece = e % (D / 4);
    if (q0 + row >= p.N) continue;
    const size_t at = (((size_t)b * p.N + q0 + row) * p.H + h) * D + piece * 4;
    const u32x2 out = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p.out_in) + at);
    const float f = sum(s_off, row) * (CAP ? sum(s_bent, row) : 1.f);
    const f32x4_t x = correct(WaveSums<D>::template get<NW>(lds0, RING, row, piece), out, f) * p.scale;
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.dq) + at) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  }
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void scored_dv_kernel(ScoredParams p) {
  using T = AttnTile<D, kTileRows>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int KS = D / 32, DB = D / 16;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ int s_first[4], s_last[4];
  const int R = p.H / p.G, g = blockIdx.x % p.G;
  const int kvt = (int)(blockIdx.x / p.G / (p.B * p.S));
  const int bs = (int)(blockIdx.x / p.G % (p.B * p.S)), b = bs % p.B, split = bs / p.B;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  const int wg0 = kvt * BKV, kv0 = wg0 + wave * 16 * KVB;

  // The query tiles from the first to the last that sees one of the workgroup's rows.
  const int tiles = (p.N + 63) / 64, halves = (p.N + 31) / 32;
  const i32x4* sees = static_cast<const i32x4*>(p.tile_sees) + (size_t)b * halves;
  // Of a 64-row tile, from its two halves; the second half of the last one may not exist.
  auto join = [](i32x4 a, i32x4 z, bool two) {
    i32x4 s = {min(a.x, z.x), max(a.y, z.y), max(a.z, z.z), min(a.w, z.w)};
    if (!two) s = i32x4{a.x, a.y, a.z, 0};
    return s;
  };
  int first = tiles, last = 0;
  for (int t = threadIdx.x; t < tiles; t += kThreads) {
    const i32x4 s = join(sees[2 * t], sees[min(2 * t + 1, halves - 1)], 2 * t + 1 < halves);
    if (s.x < wg0 + BKV && s.y > wg0) {
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

  bf16x8_t vf[KVB][KS];
#pragma unroll
  for (int kb = 0; kb < KVB; ++kb) {
    const int kv = min(kv0 + kb * 16 + fr, p.N - 1);
    const uint16_t* sv = static_cast<const uint16_t*>(p.v) + (((size_t)b * p.N + kv) * p.G + g) * D + grp * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      vf[kb][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(sv + ks * 32));
  }
  f32x4_t acc[DB][KVB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int kb = 0; kb < KVB; ++kb) acc[i][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    first = min(first, s_first[w]);
    last = max(last, s_last[w]);
  }
  first = __builtin_amdgcn_readfirstlane(first);
  last = __builtin_amdgcn_readfirstlane(last);

  // Work items: (head of the group, query tile) pairs, heads outermost; this
  // workgroup's share of them where they are split. The bounds are read as scalars
  // (an earlier kernel wrote them).
  // A split has kLeastItems items at least: under a mask the tiles differ in what they
  // have, and those with little are not split.
  const int per = max(last - first, 0);
  int it = 0, items = R * per, S = 1;
  if (p.S > 1) {
    S = max(1, min(p.S, items / kLeastItems));
    if (g == 0 && split == 0 && threadIdx.x == 0) p.tile_splits[kvt * p.B + b] = S;
    if (split >= S) return;
    it = (int)((long)items * split / S);
    items = (int)((long)items * (split + 1) / S);
  }
  typedef const __attribute__((address_space(4))) i32x4 const_i32x4;
  auto bounds = [&](int i) {
    const int t = first + i % per;
    const i32x4 a = ((const_i32x4*)sees)[2 * t], z = ((const_i32x4*)sees)[min(2 * t + 1, halves - 1)];
    return join(a, z, 2 * t + 1 < halves);
  };
  auto seek = [&](int i) {
    for (; i < items; ++i) {
      const i32x4 s = bounds(i);
      if (s.x < wg0 + BKV && s.y > wg0) break;
    }
    return i;
  };
  const size_t row_bytes = (size_t)p.H * D * 2;
  const unsigned char* gQ = static_cast<const unsigned char*>(p.q) + (size_t)b * p.N * row_bytes;
  const unsigned char* gD = static_cast<const unsigned char*>(p.dout) + (size_t)b * p.N * row_bytes;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  // An item's 64 rows' lse, Dd and seen ranges travel with its tiles, 256 bytes each.
  const uint32_t rows0 = lds0 + 4 * T::BYTES;
  auto issue = [&](int i, int stage) {
    const int lane = lane_again();
    const TileCopy<D> cp(wave, lane, row_bytes);
    const int h = g * R + i / per, r0 = (first + i % per) * kTileRows;
    const uint32_t st = lds0 + stage * 2 * T::BYTES, rs = rows0 + stage * 1024 + wave * 256;
    cp.issue(gQ + (size_t)h * D * 2, row_bytes, r0, p.N, wave, lane, st);
    cp.issue(gD + (size_t)h * D * 2, row_bytes, r0, p.N, wave, lane, st + T::BYTES);
    const uint32_t off = (uint32_t)(min(r0 + lane, p.N - 1) - r0) * 4;
    const size_t hr = ((size_t)b * p.H + h) * p.N + r0, br = (size_t)b * p.N + r0;
    const void* src = wave == 0   ? static_cast<const void*>(p.lse + hr)
                      : wave == 1 ? static_cast<const void*>(p.Dd + hr)
                      : wave == 2 ? static_cast<const void*>(p.row_lo + br)
                                  : static_cast<const void*>(p.row_hi + br);
    copy_dword_to_lds(src, off, rs);
  };
  it = seek(it);
  int stage = 0;
  if (it < items) issue(it, 0);
  while (it < items) {
    const int next = seek(it + 1);
    KL_WAIT_VMCNT(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
    if (next < items) issue(next, stage ^ 1);
    const int q0 = (first + it % per) * kTileRows, h = g * R + it / per;
    const i32x4 s = bounds(it);
    const int lane = lane_again(), fr = lane & 15, grp = lane >> 4;
    const FragOffsets<D> fi = FragOffsets<D>(fr, grp).at(lds0 + stage * 2 * T::BYTES);
    const int rows_it = (int)(rows0 + stage * 1024);
    it = next;
    stage ^= 1;
    if (s.x >= kv0 + 16 * KVB || s.y <= kv0) continue;  // no row of the tile sees this wave's
    // Rows past the end see nothing, so that a tile with a tail is an edge.
    const bool edge = s.z > kv0 || s.w < kv0 + 16 * KVB;
    const Form form(p.scale, p.cap);
    const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
#pragma unroll
    for (int qs = 0; qs < 2; ++qs) {
      u32x4 wp[KVB], wz[KVB];
      bool bad = false;  // a row that does not see a value is not finite: see the forward
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int qb = 2 * qs + hh;  // 16-row query block of the tile
        f32x4_t sc[KVB], dp[KVB];
        __builtin_amdgcn_sched_barrier(0);
        bf16x8_t aq[KS], ad[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int a = fi.s(ks) + qb * 16 * T::ROW;
          aq[ks] = lds_rows(a);
          ad[ks] = lds_rows(a + T::BYTES);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int kb = 0; kb < KVB; ++kb) {
            sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                aq[ks], vf[kb][ks], ks == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[kb], 0, 0, 0);
            dp[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                ad[ks], vf[kb][ks], ks == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : dp[kb], 0, 0, 0);
          }
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 4, 0);
#pragma unroll
        for (int ks = 0; ks + 2 < KS; ++ks) {
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2 * KVB, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 4 * KVB, 0);
        __builtin_amdgcn_sched_barrier(0);
        // Lane: query rows ql + r against value row kv0 + 16 kb + fr.
        const int ql = q0 + qb * 16 + grp * 4, rl = rows_it + (qb * 16 + grp * 4) * 4;
        auto row_data = [&](int which) {
          return *(const __attribute__((address_space(3))) f32x4_t*)(uintptr_t)(uint32_t)(rl + which * 256);
        };
        const f32x4_t lse = row_data(0), dd = row_data(1);
        int lo[4], hi[4];
        if (edge) {
          const f32x4_t a = row_data(2), z = row_data(3);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool live = ql + r < p.N;
            lo[r] = live ? __float_as_int(a[r]) : 0;
            hi[r] = live ? __float_as_int(z[r]) : 0;
          }
          bool odd = false;
#pragma unroll
          for (int kb = 0; kb < KVB; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int kv = kv0 + kb * 16 + fr;
              odd |= ((kv < lo[r]) | (kv >= hi[r])) & (not_finite(sc[kb][r]) | not_finite(dp[kb][r]));
            }
          odd = __builtin_amdgcn_ballot_w64(odd) != 0;
          bad |= odd;
          if (odd) {
#pragma unroll
            for (int kb = 0; kb < KVB; ++kb)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                sc[kb][r] = not_finite(sc[kb][r]) | not_finite(dp[kb][r]) ? __builtin_nanf("") : sc[kb][r];
          }
        }
#pragma unroll
        for (int kb = 0; kb < KVB; ++kb) {
          const float dist = (float)(ql - (kv0 + kb * 16 + fr));
          float w[4], dz[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float bend;
            weigh<Form, CAP, BIAS>(form, sc[kb][r], slope, dist + (float)r,
                                   fmaf(-lse[r], kScoredLog2e, form.C()), p.scale, w[r], bend);
            dz[r] = w[r] * (dp[kb][r] - dd[r]) * bend;
          }
          if (edge) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int kv = kv0 + kb * 16 + fr;
              const bool unseen = (kv < lo[r]) | (kv >= hi[r]);
              w[r] = unseen ? 0.f : w[r];
              dz[r] = unseen ? 0.f : dz[r];
            }
          }
          wp[kb][2 * hh] = pack2(w[0], w[1]);
          wp[kb][2 * hh + 1] = pack2(w[2], w[3]);
          wz[kb][2 * hh] = pack2(dz[0], dz[1]);
          wz[kb][2 * hh + 1] = pack2(dz[2], dz[3]);
        }
      }
      // dV^T += dO^T P + Q~^T (scale dz) over query rows 32 qs + {4 grp .., 16 + 4 grp ..}.
      __builtin_amdgcn_sched_barrier(0);
      bf16x8_t ad[DB], aq[DB];
      auto rd = [&](int db) {
        const int a = fi.t(db) + qs * 32 * T::ROW;
        ad[db] = lds_columns<T::ROW>(a + T::BYTES);
        aq[db] = lds_columns<T::ROW>(a);
        if (bad) {
          ad[db] = finite_or_zero(ad[db]);
          aq[db] = finite_or_zero(aq[db]);
        }
      };
      rd(0);
      rd(1);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        if (db + 2 < DB) rd(db + 2);
#pragma unroll
        for (int kb = 0; kb < KVB; ++kb) {
          acc[db][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              ad[db], __builtin_bit_cast(bf16x8_t, wp[kb]), acc[db][kb], 0, 0, 0);
          acc[db][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              aq[db], __builtin_bit_cast(bf16x8_t, wz[kb]), acc[db][kb], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 8, 0);
#pragma unroll
      for (int db = 0; db + 2 < DB; ++db) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2 * KVB, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 4, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 4 * KVB, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Lane holds dV^T[16 db + 4 grp + r][kv0 + 16 kb + fr]; a split leaves its sums in
  // fp32, laid out as dv.
#pragma unroll
  for (int kb = 0; kb < KVB; ++kb) {
    const int kv = kv0 + kb * 16 + fr;
    if (kv >= p.N) continue;
    const size_t at = (((size_t)b * p.N + kv) * p.G + g) * D + grp * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      if (S > 1)
        *reinterpret_cast<f32x4_t*>(p.part + (size_t)split * p.B * p.N * p.G * D + at + db * 16) = acc[db][kb];
      else
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.dv) + at + db * 16) =
            u32x2{pack2(acc[db][kb][0], acc[db][kb][1]), pack2(acc[db][kb][2], acc[db][kb][3])};
    }
  }
}

// dv of the value tiles whose sums were split, from their fp32 partial sums in split order.
__global__ __launch_bounds__(kThreads) void scored_sum_kernel(ScoredParams p) {
  const int b = blockIdx.x % p.B, kvt = blockIdx.x / p.B;
  const int S = p.tile_splits[kvt * p.B + b];
  if (S == 1) return;
  const long row = (long)p.G * p.D, n = (long)p.B * p.N * row;
  const long e = ((long)blockIdx.y * kThreads + threadIdx.x) * 4;
  if (e >= min(BKV, p.N - kvt * BKV) * row) return;
  const long at = ((long)b * p.N + kvt * BKV) * row + e;
  f32x4_t x = *reinterpret_cast<const f32x4_t*>(p.part + at);
#pragma unroll 4
  for (int s = 1; s < S; ++s) x += *reinterpret_cast<const f32x4_t*>(p.part + s * n + at);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.dv) + at) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
}

template <int D, bool CAP, bool BIAS>
hipError_t launch_form(const ScoredParams& p, hipStream_t st) {
  using T = AttnTile<D, kTileRows>;
  constexpr int dq_lds = kStages * T::BYTES;
  constexpr int dv_lds = 4 * T::BYTES + 2048;  // two stages of Q~ and dO tiles and their rows
  if (scored_few_query_tiles(p)) {
    constexpr int split_lds = 4 * 2 * AttnTile<D, 32>::BYTES;
    hipLaunchKernelGGL((scored_dq_split_kernel<D, CAP, BIAS>), dim3((unsigned)p.H * p.B * ((p.N + 31) / 32)),
                       dim3(kThreads), split_lds, st, p);
  } else {
    hipLaunchKernelGGL((scored_dq_kernel<D, CAP, BIAS>), dim3((unsigned)p.H * p.B * ((p.N + BQ - 1) / BQ)),
                       dim3(kThreads), dq_lds, st, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dv_lds > 65536) {
    static std::atomic<uint32_t> done{0};
    e = set_max_lds(reinterpret_cast<const void*>(scored_dv_kernel<D, CAP, BIAS>), dv_lds, done);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((scored_dv_kernel<D, CAP, BIAS>),
                     dim3((unsigned)p.G * p.B * p.S * ((p.N + BKV - 1) / BKV)), dim3(kThreads), dv_lds, st, p);
  e = hipGetLastError();
  if (e != hipSuccess || p.S == 1) return e;
  const dim3 grid(p.B * ((p.N + BKV - 1) / BKV), (unsigned)(((long)BKV * p.G * D / 4 + kThreads - 1) / kThreads));
  hipLaunchKernelGGL(scored_sum_kernel, grid, dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const ScoredParams& p, hipStream_t st) {
  if (p.cap > 0.f) return p.slopes ? launch_form<D, true, true>(p, st) : launch_form<D, true, false>(p, st);
  return p.slopes ? launch_form<D, false, true>(p, st) : launch_form<D, false, false>(p, st);
}

}  // namespace

hipError_t launch_scored_backward_bf16(const ScoredParams& p, hipStream_t st) {
  return p.D == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace kl
