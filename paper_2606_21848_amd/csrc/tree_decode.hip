// Drafted tokens over a value-only cache: T queries per sequence (a tree of drafted
// tokens, a chain, or the one token of a decode step) attend to the cached rows, which
// all of them see, and to the drafted rows behind them, which each sees as its word of
// the tree says. Scores with a tanh cap and a distance bias as in the scored attention.
//
// The T queries of all H / G heads of a group read the same rows, so a workgroup takes a
// block of 16 QB of these T H / G query rows over one chunk of a sequence's rows: the
// matrix cores work on whole 16-row blocks and a cached row crosses HBM once for all
// tokens and heads of a block (blocks of one chunk run side by side on one XCD where G is
// a multiple of 8, and meet its rows in L2). The four waves share the chunk's 32-row tiles, tile
// t to wave t % 4, each through a private two-stage LDS ring with no barrier, and meet
// once to merge. Only tiles that reach into the draft or past its end are masked.

#include "attn_tile.h"
#include "scored_device.h"
#include "tree_device.h"

namespace kl {
namespace {

constexpr int kThreads = 256, NW = 4;

// Copies of 32-row tiles of a cache by one wave. A tile lies in one or two pages (pages
// are at least 16 rows), so its halves have bases of their own.
template <int D, bool PAGED>
struct CacheTiles {
  using T = AttnTile<D, kTreeTile>;
  static constexpr int COPIES = T::BYTES / 1024, RPC = 1024 / T::ROW;
  uint32_t chunk[COPIES];
  int lane_row;
  const unsigned char* base;  // contiguous: the pair's first row; paged: group g of block 0
  const __attribute__((address_space(4))) int* table;
  int rows, shift, num_blocks;
  size_t block_bytes;
  __device__ __forceinline__ CacheTiles(const TreeParams& p, const TreeSpan& sp, int g, int lane)
      : lane_row(lane / T::CHUNKS), rows(sp.rows), shift(p.block_shift), num_blocks(p.num_blocks) {
#pragma unroll
    for (int c = 0; c < COPIES; ++c)
      chunk[c] = (uint32_t)(T::swz(c * RPC + lane / T::CHUNKS, lane % T::CHUNKS) * 16);
    const unsigned char* data = static_cast<const unsigned char*>(p.data);
    if constexpr (PAGED) {
      block_bytes = ((size_t)p.G << p.block_shift) * T::ROW;
      base = data + ((size_t)g << p.block_shift) * T::ROW;
      table = (const __attribute__((address_space(4))) int*)p.table + (size_t)sp.b * p.max_blocks;
    } else {
      base = data + ((size_t)sp.b * p.G + g) * p.L_max * T::ROW;
    }
  }
  // The block of row j, or -1 where there is none.
  __device__ __forceinline__ int block(int j) const {
    if constexpr (!PAGED) return 0;
    if (j >= rows) return -1;
    const int blk = table[j >> shift];
    return blk < num_blocks ? blk : -1;
  }
  // Copies the tile from row j0 on, whose halves lie in blocks b0 and b1. Rows past the
  // end are copies of the last one, halves outside the cache of some other rows.
  template <bool ONCE>
  __device__ __forceinline__ void issue(int j0, int b0, int b1, uint32_t lds) const {
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      const int half = c * RPC / 16;
      int j = j0 + 16 * half;
      const unsigned char* src;
      int last = rows - 1 - j;  // of the half, counted from its first row
      if constexpr (PAGED) {
        const int blk = half ? b1 : b0;
        // A half without a block is read from block 0; it is not used.
        src = base + (blk >= 0 ? (size_t)blk : 0) * block_bytes +
              (size_t)(j & ((1 << shift) - 1)) * T::ROW;
        last = 15;
      } else {
        if (last < 0) {
          j = rows - 1;
          last = 0;
        }
        src = base + (size_t)j * T::ROW;
      }
      const uint32_t off = (uint32_t)(min(c * RPC % 16 + lane_row, last) * T::ROW) + chunk[c];
      if constexpr (ONCE) copy_to_lds_nt(src, off, lds + c * 1024);
      else copy_to_lds(src, off, lds + c * 1024);
    }
  }
};

// The lowest n bits of a word, none for n <= 0.
__device__ __forceinline__ uint32_t below(int n) {
  return n >= 32 ? ~0u : n > 0 ? (1u << n) - 1 : 0u;
}

template <int D, int QB, bool CAP, bool BIAS, bool PAGED>
__global__ __launch_bounds__(kThreads, 2) void tree_kernel(TreeParams p) {
  constexpr int BQ = 16 * QB, KS = D / 32, DB = D / 16;
  using T = AttnTile<D, kTreeTile>;
  using Form = ScoreForm<CAP, BIAS>;
  constexpr int RING = 2 * T::BYTES;
  static_assert(RING >= BQ * D * 4, "a wave's results fit its ring");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ float s_ml[NW][BQ][2];
  __shared__ int s_depth[BIAS ? kMaxDrafts : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, grp = lane >> 4;
  const int R = p.H / p.G, M = p.T * R, blocks = (M + BQ - 1) / BQ;
  const int g = blockIdx.x % p.G, m0 = (int)(blockIdx.x / p.G % blocks) * BQ;
  const int c = blockIdx.x / p.G / blocks;
  TreeSpan sp;
  if (!tree_span(p, lane, c, -1, sp)) return;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  const uint32_t ring = lds0 + wave * RING;
  const CacheTiles<D, PAGED> cp(p, sp, g, lane);
  auto row0 = [&](int t) { return (sp.tile0 + t) * kTreeTile; };
  const bool once = blocks == 1;
  auto issue = [&](int t, int b0, int b1, int stage) {
    if (once) cp.template issue<true>(row0(t), b0, b1, ring + stage * T::BYTES);
    else cp.template issue<false>(row0(t), b0, b1, ring + stage * T::BYTES);
  };
  // Blocks of the tile at hand (now), the next one, and the one after it, whose table
  // entries are read a tile ahead of its copies.
  int now0 = -1, now1 = -1, next0 = -1, next1 = -1;
  if (wave < sp.tiles) {
    now0 = cp.block(row0(wave));
    now1 = cp.block(row0(wave) + 16);
    next0 = cp.block(row0(wave + NW));
    next1 = cp.block(row0(wave + NW) + 16);
    issue(wave, now0, now1, 0);
  }

  // Query row m0 + 16 qb + fr: token m / R of head m % R of the group.
  bf16x8_t qf[QB][KS];
  uint64_t word[QB];
  int place[QB];  // its depth
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int m = min(m0 + qb * 16 + fr, M - 1), t = m / R;
    const uint16_t* src = static_cast<const uint16_t*>(p.q) +
                          (((size_t)sp.b * p.T + t) * p.H + g * R + m % R) * D + grp * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[qb][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(src + ks * 32));
    word[qb] = tree_word(p, sp.b, t);
    place[qb] = tree_depth(word[qb], t);
  }
  float slope[QB];  // in log2 units
  if constexpr (BIAS) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
      slope[qb] = p.slopes[g * R + min(m0 + qb * 16 + fr, M - 1) % R] * kScoredLog2e;
    for (int t = threadIdx.x; t < p.T; t += kThreads) s_depth[t] = tree_depth(tree_word(p, sp.b, t), t);
    __syncthreads();
  }
  const Form form(p.scale, p.cap);
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
  for (int t = wave; t < sp.tiles; t += NW) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other stage has been read
    const int j0 = row0(t), b0 = now0, b1 = now1;
    if (t + NW < sp.tiles) {
      issue(t + NW, next0, next1, stage ^ 1);
      now0 = next0;
      now1 = next1;
      next0 = cp.block(row0(t + 2 * NW));
      next1 = cp.block(row0(t + 2 * NW) + 16);
      KL_WAIT_VMCNT(T::BYTES / 1024);
    } else {
      KL_WAIT_VMCNT(0);
    }
    asm volatile("" ::: "memory");
    const FragOffsets<D> fi = fo.at(ring + stage * T::BYTES);
    stage ^= 1;
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
    // The rows of each half end with the sequence; a half outside the cache has none.
    const int end0 = PAGED && b0 < 0 ? 0 : sp.rows, end1 = PAGED && b1 < 0 ? 0 : sp.rows;
    const bool edge = j0 + kTreeTile > min(sp.n, min(end0, end1));
    const int jl = j0 + grp * 4;
    // Bit i: this lane's query sees row j0 + 4 grp + i.
    uint32_t sees[QB];
    if (edge) {
      const uint32_t live = (below(end0 - j0) & 0xffffu) | (below(end1 - j0) & 0xffff0000u);
      const int at = sp.n - j0;  // the draft's first row in the tile
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const uint64_t w = at < 32 ? (at >= 0 ? word[qb] << at : at > -64 ? word[qb] >> -at : 0) : 0;
        sees[qb] = (((uint32_t)w | below(at)) & live) >> (grp * 4);
      }
    }
    auto unseen = [&](int qb, int kb, int r) { return (sees[qb] >> (kb * 16 + r) & 1) == 0; };
    auto bias = [&](float x, int qb, int kb, int r) -> float {
      const int j = jl + kb * 16 + r;
      int d = sp.n + place[qb] - j;
      if (edge && j >= sp.n) d = abs(place[qb] - s_depth[min(j - sp.n, p.T - 1)]);
      return fmaf(-slope[qb], (float)d, x);
    };
    const bool bad = soften<D, 2, QB>(form, sc, o, m, l, edge, unseen, bias);
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
    const int row = e / (D / 4), piece = e % (D / 4), mr = m0 + row;
    if (mr >= M) continue;
    float mm, sum;
    const f32x4_t x = merge.get(row, piece, mm, sum);
    if (sp.S == 1) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint16_t* dst = static_cast<uint16_t*>(p.out) +
                      (((size_t)sp.b * p.T + mr / R) * p.H + g * R + mr % R) * D + piece * 4;
      *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv)};
    } else {
      *reinterpret_cast<f32x4_t*>(tree_part(p, c, g, mr) + piece * 4) = x;
      if (piece == 0) {
        float* ml = tree_part_ml(p, c, g, mr);
        ml[0] = mm;
        ml[1] = sum;
      }
    }
  }
}

// Joins the chunks of a sequence, in chunk order: SUB lanes groups of D / 4 lanes per
// row, each taking every SUB-th chunk, added in a fixed order.
template <typename E, int D, int SUB>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(TreeParams p) {
  constexpr int LANES = D / 4, ROWS = kThreads / LANES / SUB;  // rows per workgroup
  __shared__ f32x4_t s_x[SUB > 1 ? kThreads : 1];
  __shared__ float s_ml[SUB > 1 ? kThreads / LANES : 1][2];
  const int lane = threadIdx.x & 63;
  const int R = p.H / p.G, M = p.T * R, blocks = (M + ROWS - 1) / ROWS;
  const int g = blockIdx.x % p.G, b = blockIdx.x / p.G / blocks;
  const int slot = threadIdx.x / LANES, piece = threadIdx.x % LANES, sub = slot % SUB;
  const int row = (int)(blockIdx.x / p.G % blocks) * ROWS + slot / SUB, m = min(row, M - 1);
  TreeSpan sp;
  if (!tree_span(p, lane, 0, b, sp) || sp.S == 1) return;
  float mm = -INFINITY, sum = 0.f;
  f32x4_t x = {0.f, 0.f, 0.f, 0.f};
  auto take = [&](float mk, float lk, f32x4_t xk) {
    const float mn = fmaxf(mm, mk), ms = mn == -INFINITY ? 0.f : mn;
    const float f = fast_exp2(mm - ms), fk = fast_exp2(mk - ms);
    mm = mn;
    sum = sum * f + lk * fk;
    x = x * f + xk * fk;
  };
#pragma unroll 4
  for (int s = sub; s < sp.S; s += SUB) {
    const float* ml = tree_part_ml(p, sp.first + s, g, m);
    take(ml[0], ml[1], *reinterpret_cast<const f32x4_t*>(tree_part(p, sp.first + s, g, m) + piece * 4));
  }
  if constexpr (SUB > 1) {
    s_x[threadIdx.x] = x;
    if (piece == 0) {
      s_ml[slot][0] = mm;
      s_ml[slot][1] = sum;
    }
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int k = 1; k < SUB; ++k) take(s_ml[slot + k][0], s_ml[slot + k][1], s_x[threadIdx.x + k * LANES]);
  }
  if (row >= M) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const size_t at = (((size_t)b * p.T + m / R) * p.H + g * R + m % R) * D + piece * 4;
  if constexpr (sizeof(E) == 2)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) =
        u32x2{pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv)};
  else
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = x * inv;
}

template <int D, int QB, bool CAP, bool BIAS, bool PAGED>
hipError_t launch_tree(const TreeParams& p, hipStream_t st) {
  constexpr int lds = NW * 2 * AttnTile<D, kTreeTile>::BYTES;
  const unsigned blocks = (p.T * (p.H / p.G) + 16 * QB - 1) / (16 * QB);
  hipLaunchKernelGGL((tree_kernel<D, QB, CAP, BIAS, PAGED>), dim3((p.chunks + p.B) * blocks * p.G),
                     dim3(kThreads), lds, st, p);
  return hipGetLastError();
}

template <int D, int QB>
hipError_t launch_qb(const TreeParams& p, hipStream_t st) {
  auto layout = [&](auto cap, auto bias) {
    return p.paged ? launch_tree<D, QB, decltype(cap)::value, decltype(bias)::value, true>(p, st)
                   : launch_tree<D, QB, decltype(cap)::value, decltype(bias)::value, false>(p, st);
  };
  using Y = std::true_type;
  using N = std::false_type;
  if (p.cap > 0.f) return p.slopes ? layout(Y{}, Y{}) : layout(Y{}, N{});
  return p.slopes ? layout(N{}, Y{}) : layout(N{}, N{});
}

template <typename E, int D>
hipError_t launch_merge(const TreeParams& p, hipStream_t st) {
  const int M = p.T * (p.H / p.G);
  // Few rows: eight groups of lanes share a row's chunks (batch 1 has many of them).
  if ((long)p.B * p.G * M <= 1024) {
    constexpr int SUB = 8, ROWS = kThreads / (D / 4) / SUB;
    hipLaunchKernelGGL((tree_merge_kernel<E, D, SUB>), dim3(p.B * p.G * ((M + ROWS - 1) / ROWS)),
                       dim3(kThreads), 0, st, p);
  } else {
    constexpr int ROWS = kThreads / (D / 4);
    hipLaunchKernelGGL((tree_merge_kernel<E, D, 1>), dim3(p.B * p.G * ((M + ROWS - 1) / ROWS)),
                       dim3(kThreads), 0, st, p);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const TreeParams& p, hipStream_t st) {
  const hipError_t e = p.T * (p.H / p.G) <= 16 ? launch_qb<D, 1>(p, st) : launch_qb<D, 2>(p, st);
  return e != hipSuccess || !p.part ? e : launch_tree_merge(p, st);
}

}  // namespace

hipError_t launch_tree_merge(const TreeParams& p, hipStream_t st) {
  if (p.dtype == KL_BF16) return p.D == 128 ? launch_merge<uint16_t, 128>(p, st) : launch_merge<uint16_t, 64>(p, st);
  return p.D == 128 ? launch_merge<float, 128>(p, st) : launch_merge<float, 64>(p, st);
}

hipError_t launch_tree_decode_bf16(const TreeParams& p, hipStream_t st) {
  return p.D == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace kl
