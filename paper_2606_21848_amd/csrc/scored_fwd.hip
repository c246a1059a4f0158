// Scored keyless attention, bf16 forward on the matrix cores: the keyless attention
// (S^T = V Q~^T, then O^T += V^T P^T from one tile of values in LDS) with a tanh cap
// and a distance bias on the scores and a range of seen value rows per query.
//
// A workgroup (4 waves) owns 64 QB query rows of one head, a wave 16 QB of them. It
// walks the 64-row value tiles that any of its rows sees, in order, three in flight
// (direct-to-LDS copies); a wave passes over a tile that none of its rows sees, and
// masks only in tiles that some of its rows see in part. Each lane keeps the ranges
// of its QB queries in registers, so documents, prefixes, windows and padding cost
// what the causal mask costs.
//
// The routed queries are not multiplied by the scale (that would round them once
// more): the scale joins the exponent's multiply-add. The weights' sum is taken from
// the unrounded weights, in fp32, since the backward pass forms P from it; the weights are
// rounded to bf16 once, as the second product's operand.
//
// 8192 tokens, 32 heads on 8 groups of 128, causal, cap 50: 615 us, 0.89 PFLOP/s. Matrix
// instructions take 36% of the cycles and the vector ones of the softmax (an exponential
// and a reciprocal for the cap, an exponential for the weight) 59%, and the two hardly
// overlap: an instruction of one wave does not start while the other wave's occupies the
// issue. Interleaving them by hand spilled 50 registers and more (840 us).

#include <type_traits>

#include "attn_tile.h"
#include "scored_device.h"

namespace kl {
namespace {

constexpr int kThreads = 256;
constexpr int kTileRows = 64;  // value rows per tile
constexpr int kStages = 3;     // tiles in LDS
template <int D, int QB, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void scored_fwd_kernel(ScoredParams p) {
  using T = AttnTile<D, kTileRows>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int WQ = 16 * QB, BQ = 4 * WQ, KS = D / 32, DB = D / 16;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ int s_any[4][2];
  const HeadTile ht(p, BQ);
  const int h = ht.h, g = ht.g, b = ht.b, qt = ht.qt;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  const int q0 = qt * BQ + wave * WQ;

  SeenRange seen[QB];
  SeenBounds sb;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    seen[qb] = seen_range(p, b, min(q0 + qb * 16 + fr, p.N - 1));
    sb.add(seen[qb]);
  }
  sb.over_rows();
  sb.make_uniform();
  if (q0 >= p.N) sb.any_lo = sb.any_hi = 0;  // rows past the end: this wave only copies
  if (lane == 0) {
    s_any[wave][0] = sb.any_hi > sb.any_lo ? sb.any_lo : 0x7fffffff;
    s_any[wave][1] = sb.any_hi;
  }
  __syncthreads();
  int lo = s_any[0][0], hi = s_any[0][1];
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    lo = min(lo, s_any[w][0]);
    hi = max(hi, s_any[w][1]);
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

  bf16x8_t qf[QB][KS];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const uint16_t* src = static_cast<const uint16_t*>(p.q) +
                          (((size_t)b * p.N + min(q0 + qb * 16 + fr, p.N - 1)) * p.H + h) * D + grp * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[qb][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(src + ks * 32));
  }
  const Form form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  f32x4_t o[DB][QB];
  float m[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = -INFINITY;
    l[qb] = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const FragOffsets<D> fo(fr, grp);
  // The wait for the queries is taken here, where the first tiles are awaited anyway.
  KL_WAIT_VMCNT(0);
  int stage = 0;
  for (int t = 0; t < ntiles; ++t) {
    if (t + 1 < ntiles) KL_WAIT_VMCNT((kStages - 2) * T::COPIES);
    else KL_WAIT_VMCNT(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage refilled below has been read
    __syncthreads();
    if (t + kStages - 1 < ntiles) issue(t + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
    const int j0 = (t0 + t) * kTileRows;
    const int tile = (int)lds0 + stage * T::BYTES;
    stage = stage == kStages - 1 ? 0 : stage + 1;
    if (j0 >= sb.any_hi || j0 + kTileRows <= sb.any_lo) continue;
    const FragOffsets<D> fi = fo.at(tile);
    f32x4_t sc[4][QB];
    {
      int offS[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) offS[ks] = fi.s(ks);
      bf16x8_t sa[2][KS];
      auto rows = [&](int kb, int ks) { return lds_rows(offS[ks] + kb * 16 * T::ROW); };
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sa[0][ks] = rows(0, ks);
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        if (kb + 1 < 4) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) sa[(kb + 1) & 1][ks] = rows(kb + 1, ks);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            sc[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                sa[kb & 1][ks], qf[qb][ks], ks == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[kb][qb], 0, 0, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedDsRead, KS, 0);
#pragma unroll
      for (int kb = 0; kb < 3; ++kb) {
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, KS, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, KS * QB, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, KS * QB, 0);
    }
    const bool edge = j0 < sb.all_lo || j0 + kTileRows > sb.all_hi;
    const int jl = j0 + grp * 4;
    const bool bad = soften<D, 4, QB>(
        form, sc, o, m, l, edge,
        [&](int qb, int kb, int r) {
          const int j = jl + kb * 16 + r;
          return (j < seen[qb].lo) | (j >= seen[qb].hi);
        },
        [&](float x, int qb, int kb, int r) {
          return fmaf(-slope, fabsf((float)(q0 + qb * 16 + fr - jl) - (float)(kb * 16 + r)), x);
        });
    int offT[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) offT[db] = fi.t(db);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8_t pf[QB], av[DB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) pf[qb] = pack8(sc[2 * ks][qb], sc[2 * ks + 1][qb]);
#pragma unroll
      for (int db = 0; db < DB; ++db) av[db] = lds_columns<T::ROW>(offT[db] + ks * 32 * T::ROW);
      if (bad) {
#pragma unroll
        for (int db = 0; db < DB; ++db) av[db] = finite_or_zero(av[db]);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[db], pf[qb], o[db][qb], 0, 0, 0);
    }
  }

  // Lane holds O[q][16 db + 4 grp + r]; the sums of a query lie over its four lane groups.
  uint16_t* __restrict__ O = static_cast<uint16_t*>(p.out);
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int q = q0 + qb * 16 + fr;
    float sum = l[qb] + __shfl_xor(l[qb], 16);
    sum += __shfl_xor(sum, 32);
    if (q >= p.N) continue;
    const bool none = seen[qb].lo >= seen[qb].hi;
    const float inv = none ? 0.f : 1.f / sum;
    if (p.lse && grp == 0)
      p.lse[((size_t)b * p.H + h) * p.N + q] = none ? -INFINITY : (m[qb] + __log2f(sum)) * kScoredLn2;
    const size_t at = (((size_t)b * p.N + q) * p.H + h) * D + grp * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const f32x4_t x = o[db][qb] * inv;
      if (p.out_f32) *reinterpret_cast<f32x4_t*>(p.out_f32 + at + db * 16) = x;
      *reinterpret_cast<u32x2*>(O + at + db * 16) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    }
  }
}

// The same for few query tiles (short prompts, few heads): a workgroup owns 32 query rows
// of one head and its four waves share the 32-row value tiles, tile t to wave t % 4, each
// through a private two-stage ring with no barrier, and meet once to merge. 517 tokens, 12
// heads, prefix mask, cap 30: 10.2 us, the latency of a few tiles and of the merge.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void scored_fwd_split_kernel(ScoredParams p) {
  constexpr int QB = 2, NW = 4, RV = 32, BQ = 16 * QB, KS = D / 32, DB = D / 16;
  using T = AttnTile<D, RV>;
  using Copier = WaveCopier<D, RV>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int RING = 2 * T::BYTES;
  static_assert(RING == BQ * D * 4, "a wave's results fit its ring");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ float s_ml[NW][BQ][2];
  const HeadTile ht(p, BQ);
  const int h = ht.h, g = ht.g, b = ht.b, q0 = ht.qt * BQ;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  SeenRange seen[QB];
  SeenBounds sb;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    seen[qb] = seen_range(p, b, min(q0 + qb * 16 + fr, p.N - 1));
    sb.add(seen[qb]);
  }
  sb.over_rows();
  sb.make_uniform();
  const bool any = sb.any_lo < sb.any_hi;
  const int t0 = any ? sb.any_lo / RV : 0, tend = any ? (sb.any_hi + RV - 1) / RV : 0;

  const size_t row_bytes = (size_t)p.G * D * 2;
  const unsigned char* gV = static_cast<const unsigned char*>(p.v) + ((size_t)b * p.N * p.G + g) * D * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  const uint32_t ring = lds0 + wave * RING;
  const Copier cp(lane, row_bytes);
  if (t0 + wave < tend) cp.issue(gV, row_bytes, (t0 + wave) * RV, p.N, lane, ring);
  bf16x8_t qf[QB][KS];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const uint16_t* src = static_cast<const uint16_t*>(p.q) +
                          (((size_t)b * p.N + min(q0 + qb * 16 + fr, p.N - 1)) * p.H + h) * D + grp * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[qb][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(src + ks * 32));
  }
  const Form form(p.scale, p.cap);
  const float slope = BIAS ? p.slopes[h] * kScoredLog2e : 0.f;
  f32x4_t o[DB][QB];
  float m[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = -INFINITY;
    l[qb] = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
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
    const int j0 = t * RV;
    const FragOffsets<D> fi = fo.at(ring + stage * T::BYTES);
    stage ^= 1;
    if (j0 >= sb.any_hi || j0 + RV <= sb.any_lo) continue;
    f32x4_t sc[2][QB];
    bf16x8_t sa[2][KS];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sa[kb][ks] = lds_rows(fi.s(ks) + kb * 16 * T::ROW);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          sc[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              sa[kb][ks], qf[qb][ks], ks == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[kb][qb], 0, 0, 0);
    const int jl = j0 + grp * 4;
    const bool bad = soften<D, 2, QB>(
        form, sc, o, m, l, j0 < sb.all_lo || j0 + RV > sb.all_hi,
        [&](int qb, int kb, int r) {
          const int j = jl + kb * 16 + r;
          return (j < seen[qb].lo) | (j >= seen[qb].hi);
        },
        [&](float x, int qb, int kb, int r) {
          return fmaf(-slope, fabsf((float)(q0 + qb * 16 + fr - jl) - (float)(kb * 16 + r)), x);
        });
    bf16x8_t pf[QB], av[DB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) pf[qb] = pack8(sc[0][qb], sc[1][qb]);
#pragma unroll
    for (int db = 0; db < DB; ++db) av[db] = lds_columns<T::ROW>(fi.t(db));
    if (bad) {
#pragma unroll
      for (int db = 0; db < DB; ++db) av[db] = finite_or_zero(av[db]);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
        o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[db], pf[qb], o[db][qb], 0, 0, 0);
  }
  WaveMerge<D, QB, NW> merge(s_ml, lds0, RING, wave, fr, grp);
  merge.put(m, l, o);
  for (int e = threadIdx.x; e < BQ * D / 4; e += kThreads) {
    const int row = e / (D / 4), piece = e % (D / 4);
    if (q0 + row >= p.N) continue;
    float mm, sum;
    f32x4_t x = merge.get(row, piece, mm, sum);
    const bool none = sum == 0.f;
    x *= none ? 0.f : 1.f / sum;
    const size_t at = (((size_t)b * p.N + q0 + row) * p.H + h) * D + piece * 4;
    const size_t lrow = ((size_t)b * p.H + h) * p.N + q0 + row;
    if (p.lse && piece == 0) p.lse[lrow] = none ? -INFINITY : (mm + __log2f(sum)) * kScoredLn2;
    if (p.out_f32) *reinterpret_cast<f32x4_t*>(p.out_f32 + at) = x;
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  }
}

template <int D, int QB, bool CAP, bool BIAS>
hipError_t launch_qb(const ScoredParams& p, hipStream_t st) {
  constexpr int BQ = 64 * QB, lds = kStages * AttnTile<D, kTileRows>::BYTES;
  const dim3 grid((unsigned)p.H * p.B * ((p.N + BQ - 1) / BQ));
  hipLaunchKernelGGL((scored_fwd_kernel<D, QB, CAP, BIAS>), grid, dim3(kThreads), lds, st, p);
  return hipGetLastError();
}

template <int D, bool CAP, bool BIAS>
hipError_t launch_form(const ScoredParams& p, hipStream_t st) {
  if (scored_few_query_tiles(p)) {
    constexpr int lds = 4 * 2 * AttnTile<D, 32>::BYTES;
    hipLaunchKernelGGL((scored_fwd_split_kernel<D, CAP, BIAS>), dim3((unsigned)p.H * p.B * ((p.N + 31) / 32)),
                       dim3(kThreads), lds, st, p);
    return hipGetLastError();
  }
  return launch_qb<D, 2, CAP, BIAS>(p, st);
}

template <int D>
hipError_t launch_d(const ScoredParams& p, hipStream_t st) {
  if (p.cap > 0.f) return p.slopes ? launch_form<D, true, true>(p, st) : launch_form<D, true, false>(p, st);
  return p.slopes ? launch_form<D, false, true>(p, st) : launch_form<D, false, false>(p, st);
}

}  // namespace

// Whether the kernels of 128 query rows per workgroup would leave some of the chip's 512
// places empty; then a workgroup's waves share 32 rows' value tiles. Causal, d_head 128, us:
// forward 24.8 against 30.0 with 256 such workgroups (32 heads, 1024 rows), 71 against 95
// with 384 (12 heads, 4000 rows), 59 against 53 with 512 (32 heads, 2000 rows); training
// 114 against 124, 287 against 338 and 240 against 225.
bool scored_few_query_tiles(const ScoredParams& p) {
  const long heads = (long)p.H * p.B;
  return heads * ((p.N + 127) / 128) < 512;
}

hipError_t launch_scored_forward_bf16(const ScoredParams& p, hipStream_t st) {
  return p.D == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace kl
