// Drafted tokens over a value-only cache: T queries per sequence (a tree of drafted
// tokens, a chain, or the one token of a decode step) attend to the cached rows, which
// all of them see, and to the drafted rows behind them, which each sees as its word of
// the tree says. Scores with a tanh cap and a distance bias as in the scored attention.
//
// The T queries of all H / G heads of a group read the same rows, so a workgroup takes a
// block of these T H / G query rows over a piece of the cache: the matrix cores work on
// whole 16-row blocks and a cached row crosses HBM once for all tokens and heads of a
// block (blocks of one piece run side by side on one XCD where G is a multiple of 8, and
// meet its rows in L2). Only tiles that reach into the draft or past its end are masked.
// The weights are rounded to bf16 once, as the second product's operand; their sum is not.
//
// 16 trees of 16 tokens, 32 heads on 8 groups of 128, paged caches of 1k to 32k rows, cap
// 50: 106 us, 3.0 TB/s of the cache and 0.38 PFLOP/s (100 and a merge of 5): the vector
// instructions of the softmax for 64 query rows, at one 8-wave workgroup per CU; the copies
// alone take 63. 8 trees of 64 tokens, 32 heads on 32 groups, 2k to 4k rows: 65 us, 3.1 TB/s.

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
  __device__ __forceinline__ CacheTiles(const TreeParams& p, const TreeSeg& sp, int g, int lane)
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
  // Copies the given part of the tile from row j0 on (HALF: its rows 16 HALF .. + 15),
  // which lies in block blk. Rows past the end are copies of the last one, a half outside
  // the cache is some other rows.
  template <int HALF>
  __device__ __forceinline__ void issue(int j0, int blk, bool once, uint32_t lds) const {
    int j = j0 + 16 * HALF;
    const unsigned char* src;
    int last = rows - 1 - j;  // of the half, counted from its first row
    if constexpr (PAGED) {
      // A half without a block is read from block 0; it is not used.
      src = base + (blk >= 0 ? (size_t)blk : 0) * block_bytes + (size_t)(j & ((1 << shift) - 1)) * T::ROW;
      last = 15;
    } else {
      if (last < 0) {
        j = rows - 1;
        last = 0;
      }
      src = base + (size_t)j * T::ROW;
    }
#pragma unroll
    for (int c = HALF * COPIES / 2; c < (HALF + 1) * COPIES / 2; ++c) {
      const uint32_t off = (uint32_t)(min(c * RPC % 16 + lane_row, last) * T::ROW) + chunk[c];
      if (once) copy_to_lds_nt(src, off, lds + c * 1024);
      else copy_to_lds(src, off, lds + c * 1024);
    }
  }
};

// The lowest n bits of a word, none for n <= 0.
__device__ __forceinline__ uint32_t below(int n) {
  return n >= 32 ? ~0u : n > 0 ? (1u << n) - 1 : 0u;
}

// The query rows of a wave and their running results: rows m0 + 16 qb + fr of the T H / G
// rows of a (sequence, group), row m being token m / R of head m % R of the group.
template <int D, int QB, bool CAP, bool BIAS>
struct TreeRows {
  static constexpr int KS = D / 32, DB = D / 16;
  using T = AttnTile<D, kTreeTile>;
  using Form = ScoreForm<CAP, BIAS>;
  bf16x8_t qf[QB][KS];
  uint64_t word[QB];
  int place[QB];    // depth
  float slope[QB];  // in log2 units
  f32x4_t o[DB][QB];
  float m[QB], l[QB];
  __device__ __forceinline__ void load(const TreeParams& p, int b, int g, int R, int M, int m0, int fr, int grp) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int row = min(m0 + qb * 16 + fr, M - 1), t = row / R, r = row - t * R;
      const uint16_t* src =
          static_cast<const uint16_t*>(p.q) + (((size_t)b * p.T + t) * p.H + g * R + r) * D + grp * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        qf[qb][ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(src + ks * 32));
      word[qb] = tree_word(p, b, t);
      place[qb] = tree_depth(word[qb], t);
      if constexpr (BIAS) slope[qb] = p.slopes[g * R + r] * kScoredLog2e;
      m[qb] = -INFINITY;
      l[qb] = 0.f;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
  // One landed tile, whose first row is j0 and whose halves end at rows end0 and end1.
  __device__ __forceinline__ void take(const Form& form, const FragOffsets<D>& fi, const TreeParams& p,
                                       const TreeSeg& sp, int j0, int end0, int end1, const int* s_depth,
                                       int grp) {
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
};

// Stores four columns of a merged row: the output where the segment is the whole
// sequence, else the slot's partial result.
template <int D>
__device__ __forceinline__ void tree_store(const TreeParams& p, const TreeSeg& sp, int g, int R, int mr, int piece,
                                           f32x4_t x, float mm, float sum) {
  if (sp.whole) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int t = mr / R;
    uint16_t* dst =
        static_cast<uint16_t*>(p.out) + (((size_t)sp.b * p.T + t) * p.H + g * R + mr - t * R) * D + piece * 4;
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv)};
  } else {
    *reinterpret_cast<f32x4_t*>(tree_part(p, sp.slot, g, mr) + piece * 4) = x;
    if (piece == 0) {
      float* ml = tree_part_ml(p, sp.slot, g, mr);
      ml[0] = mm;
      ml[1] = sum;
    }
  }
}

// NB blocks of 16 QB query rows per workgroup, four waves each. The four waves of a block
// share a segment's 32-row tiles, tile t to wave t % 4. With one block a wave's tiles come
// through a private two-stage ring with no barrier. With two, the waves of both blocks
// work on the same four tiles at a time, each wave having copied one half tile, through
// four common stages with one barrier per four tiles: a cached row is copied once for all
// 32 QB rows, where two workgroups of one block each copied it twice (16 x 16 tokens, 32
// heads on 8 groups, 1k to 32k rows: 105 us against 111).
template <int D, int QB, int NB, bool CAP, bool BIAS, bool PAGED>
__global__ __launch_bounds__(NB * 256, NB == 1 ? 2 : 1) void tree_kernel(TreeParams p) {
  constexpr int BQ = 16 * QB;
  using T = AttnTile<D, kTreeTile>;
  constexpr int STAGES = NB == 1 ? 2 : 4;
  constexpr int RESULT = BQ * D * 4;  // a wave's results
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ float s_ml[NB][NW][BQ][2];
  __shared__ int s_depth[BIAS ? kMaxDrafts : 1];
  const int lane = threadIdx.x & 63;
  const int wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = wave8 % NW, rb = wave8 / NW;
  const int fr = lane & 15, grp = lane >> 4;
  const int R = p.H / p.G, M = p.T * R, blocks = (M + NB * BQ - 1) / (NB * BQ);
  const int g = blockIdx.x % p.G, w0 = (int)(blockIdx.x / p.G % blocks) * (NB * BQ), m0 = w0 + rb * BQ;
  const int c = blockIdx.x / p.G / blocks;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)smem;
  const bool once = blocks == 1;
  const ScoreForm<CAP, BIAS> form(p.scale, p.cap);
  const FragOffsets<D> fo(fr, grp);
  TreeWalk walk(p, lane, c);
  TreeSeg sp;
  while (walk.next(p, lane, sp)) {
    const CacheTiles<D, PAGED> cp(p, sp, g, lane);
    auto row0 = [&](int t) { return (sp.tile0 + t) * kTreeTile; };
    auto end_of = [&](int blk) { return PAGED && blk < 0 ? 0 : sp.rows; };
    TreeRows<D, QB, CAP, BIAS> rows;
    if constexpr (NB == 1) {
      const uint32_t ring = lds0 + wave * (2 * T::BYTES);
      auto issue = [&](int t, int b0, int b1, int stage) {
        cp.template issue<0>(row0(t), b0, once, ring + stage * T::BYTES);
        cp.template issue<1>(row0(t), b1, once, ring + stage * T::BYTES);
      };
      // Blocks of the tile at hand and of the next one, read a tile ahead of its copies.
      int now0 = -1, now1 = -1, next0 = -1, next1 = -1;
      if (wave < sp.tiles) {
        now0 = cp.block(row0(wave));
        now1 = cp.block(row0(wave) + 16);
        next0 = cp.block(row0(wave + NW));
        next1 = cp.block(row0(wave + NW) + 16);
        issue(wave, now0, now1, 0);
      }
      rows.load(p, sp.b, g, R, M, m0, fr, grp);
      if constexpr (BIAS) {
        for (int t = threadIdx.x; t < p.T; t += NB * 256) s_depth[t] = tree_depth(tree_word(p, sp.b, t), t);
        __syncthreads();
      }
      int stage = 0;
      for (int t = wave; t < sp.tiles; t += NW) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other stage has been read
        const int b0 = now0, b1 = now1;
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
        rows.take(form, fo.at(ring + stage * T::BYTES), p, sp, row0(t), end_of(b0), end_of(b1), s_depth, grp);
        stage ^= 1;
      }
    } else {
      // Step i takes tiles 4 i .. 4 i + 3 from stage i % 4; this wave copies half rb of
      // tile 4 i + wave and takes that tile.
      constexpr int AHEAD = STAGES - 1, COPIES = T::BYTES / 2048;
      const int steps = (sp.tiles + NW - 1) / NW;
      int blk[AHEAD + 1][2];  // blocks of the halves of this wave's tiles of steps i .. i + 3
      auto look = [&](int i, int (&x)[2]) {
        x[0] = cp.block(row0(NW * i + wave));
        x[1] = cp.block(row0(NW * i + wave) + 16);
      };
      auto issue = [&](int i, const int (&x)[2]) {
        const int t = NW * i + wave;
        const uint32_t at = lds0 + ((i % STAGES) * NW + wave) * T::BYTES;
        // A step's last tiles may not exist: their rows are copies of the last one.
        if (rb == 0) cp.template issue<0>(row0(t), x[0], once, at);
        else cp.template issue<1>(row0(t), x[1], once, at);
      };
#pragma unroll
      for (int i = 0; i <= AHEAD; ++i) look(i, blk[i]);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i < steps) issue(i, blk[i]);
      rows.load(p, sp.b, g, R, M, m0, fr, grp);
      if constexpr (BIAS)
        for (int t = threadIdx.x; t < p.T; t += NB * 256) s_depth[t] = tree_depth(tree_word(p, sp.b, t), t);
      KL_WAIT_VMCNT(0);
      for (int i = 0; i < steps; ++i) {
        const int ahead = min(AHEAD - 1, steps - 1 - i);  // steps issued after this one
        if (ahead == 2) KL_WAIT_VMCNT(2 * COPIES);
        else if (ahead == 1) KL_WAIT_VMCNT(COPIES);
        else KL_WAIT_VMCNT(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage refilled below has been read
        __syncthreads();
        if (i + AHEAD < steps) issue(i + AHEAD, blk[AHEAD]);
        const int t = NW * i + wave, b0 = blk[0][0], b1 = blk[0][1];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          blk[k][0] = blk[k + 1][0];
          blk[k][1] = blk[k + 1][1];
        }
        look(i + AHEAD + 1, blk[AHEAD]);
        if (t < sp.tiles)
          rows.take(form, fo.at(lds0 + ((i % STAGES) * NW + wave) * T::BYTES), p, sp, row0(t), end_of(b0),
                    end_of(b1), s_depth, grp);
      }
    }
    WaveMerge<D, QB, NW> merge(s_ml[rb], lds0 + rb * NW * RESULT, RESULT, wave, fr, grp);
    merge.put(rows.m, rows.l, rows.o);
    for (int e = threadIdx.x; e < NB * BQ * D / 4; e += NB * 256) {
      const int row = e / (D / 4), piece = e % (D / 4), mr = w0 + row, k = row / BQ;
      if (mr >= M) continue;
      const WaveMerge<D, QB, NW> from(s_ml[k], lds0 + k * NW * RESULT, RESULT, wave, fr, grp);
      float mm, sum;
      const f32x4_t x = from.get(row - k * BQ, piece, mm, sum);
      tree_store<D>(p, sp, g, R, mr, piece, x, mm, sum);
    }
    __syncthreads();  // the results have been read: the next segment may fill their place
  }
}

// Joins a sequence's partial results, in slot order: SUB groups of D / 4 lanes per row,
// each taking every SUB-th slot, added in a fixed order.
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
  int first;
  const int count = tree_slots(p, lane, b, first);
  if (count == 1) return;
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
  for (int s = sub; s < count; s += SUB) {
    const float* ml = tree_part_ml(p, first + s, g, m);
    take(ml[0], ml[1], *reinterpret_cast<const f32x4_t*>(tree_part(p, first + s, g, m) + piece * 4));
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

template <int D, int QB, int NB, bool CAP, bool BIAS, bool PAGED>
hipError_t launch_tree(const TreeParams& p, hipStream_t st) {
  constexpr int tile = AttnTile<D, kTreeTile>::BYTES;
  constexpr int results = NB * NW * 16 * QB * D * 4, stages = NB == 1 ? NW * 2 * tile : NW * 4 * tile;
  constexpr int lds = results > stages ? results : stages;
  const unsigned blocks = (p.T * (p.H / p.G) + 16 * QB * NB - 1) / (16 * QB * NB);
  if (lds > 65536) {
    static std::atomic<uint32_t> done{0};
    const hipError_t e =
        set_max_lds(reinterpret_cast<const void*>(tree_kernel<D, QB, NB, CAP, BIAS, PAGED>), lds, done);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((tree_kernel<D, QB, NB, CAP, BIAS, PAGED>),
                     dim3((unsigned)p.chunks * (p.per > 0 ? p.B : 1) * blocks * p.G), dim3(NB * 256), lds, st, p);
  return hipGetLastError();
}

template <int D, int QB, int NB>
hipError_t launch_qb(const TreeParams& p, hipStream_t st) {
  auto layout = [&](auto cap, auto bias) {
    return p.paged ? launch_tree<D, QB, NB, decltype(cap)::value, decltype(bias)::value, true>(p, st)
                   : launch_tree<D, QB, NB, decltype(cap)::value, decltype(bias)::value, false>(p, st);
  };
  using Y = std::true_type;
  using N = std::false_type;
  if (p.cap > 0.f) return p.slopes ? layout(Y{}, Y{}) : layout(Y{}, N{});
  return p.slopes ? layout(N{}, Y{}) : layout(N{}, N{});
}

template <typename E, int D>
hipError_t launch_merge(const TreeParams& p, hipStream_t st) {
  const int M = p.T * (p.H / p.G);
  // Few rows: eight groups of lanes share a row's pieces (a batch of one has many of them:
  // 4 tokens, 30000 rows, 32 heads on 8 groups, 18.0 us in all against 21.7 of one group;
  // with 1024 rows in 4 sequences 32.8 against 33.1, with 2048 39.0 against 37.9).
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
  const hipError_t e = p.block_rows == 16   ? launch_qb<D, 1, 1>(p, st)
                       : p.block_rows == 32 ? launch_qb<D, 2, 1>(p, st)
                                            : launch_qb<D, 2, 2>(p, st);
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
