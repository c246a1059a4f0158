// 16-row blocks of fp32 matrices on v_mfma_f32_16x16x4_f32, shared by the fp32 attention
// kernels. A row block is read from memory straight into the first operand's layout (lane
// (r, g) = (lane % 16, lane / 16) holds columns 16 s + 4 g .. + 3 of row r); scores come
// out with one own row per lane column and the other block's rows 4 g + i in register i,
// the second product's second operand as it stands; its first operand, the other block
// transposed, is read from an LDS copy with row pitch D + 4 floats.
#pragma once

#include <hip/hip_runtime.h>

#include "kl_device.h"

namespace kl {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

template <int D>
struct Block {  // a 16-row block staged by one wave
  static constexpr int S = D / 16;      // 16-byte pieces per lane
  static constexpr int PITCH = D + 4;   // floats
  static constexpr int FLOATS = 16 * PITCH;
};

// Row `row` (zeros when it is not below `rows`) of a [rows, ...] matrix, in the
// layout above.
template <int D>
__device__ __forceinline__ void load_rows(const float* base, long stride, int row, int rows, int g,
                                          f32x4_t (&v)[D / 16]) {
  const bool live = row < rows;
  const float* src = base + (size_t)(live ? row : 0) * stride + 4 * g;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(src + 16 * s);
    v[s] = live ? x : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
}

template <int D>
__device__ __forceinline__ void stage_rows(float* tile, int r, int g, const f32x4_t (&v)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    *reinterpret_cast<f32x4_t*>(tile + r * Block<D>::PITCH + 16 * s + 4 * g) = v[s];
}

// acc[a row][b row] += sum over the D columns.
template <int D>
__device__ __forceinline__ f32x4_t dot_rows(const f32x4_t (&a)[D / 16], const f32x4_t (&b)[D / 16],
                                            f32x4_t acc) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][j], b[s][j], acc, 0, 0, 0);
  return acc;
}

// acc[db] (columns 16 db + 4 g + i of the result, own row r) += tile^T w over
// the tile's 16 rows.
template <int D>
__device__ __forceinline__ void add_weighted(const float* tile, int r, int g, f32x4_t w,
                                             f32x4_t (&acc)[D / 16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
      acc[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(
          tile[(4 * g + i) * Block<D>::PITCH + 16 * db + r], w[i], acc[db], 0, 0, 0);
}

// The same on a diagonal block that holds an infinity or a NaN: rows the own row
// does not see (`first` .. `last` are seen) must not reach it, not even as 0 x inf.
template <int D>
__device__ __forceinline__ void add_weighted_seen(const float* tile, int r, int g, f32x4_t w,
                                                  int first, int last, f32x4_t (&acc)[D / 16]) {
#pragma unroll 1
  for (int k = 0; k < 16; ++k) {
    const float x = (k & 2) ? ((k & 1) ? w[3] : w[2]) : ((k & 1) ? w[1] : w[0]);
    const float wk = __shfl(x, (k >> 2) * 16 + r, 64);
    const bool seen = k >= first && k <= last;
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = tile[k * Block<D>::PITCH + 16 * db + 4 * g + i];
        acc[db][i] = seen ? fmaf(wk, v, acc[db][i]) : acc[db][i];
      }
  }
}

template <int D>
__device__ __forceinline__ bool any_not_finite(const f32x4_t (&v)[D / 16]) {
  bool bad = false;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) bad |= !(fabsf(v[s][j]) < INFINITY);
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}

// Sums the waves' acc (scaled by `f`) into out(row, column, value) calls, one
// per element of the 16 x D result, in wave order. Uses every wave's tile.
template <int D, int NW, class Out>
__device__ __forceinline__ void merge_sum(float* lds, float* tile, int r, int g, float f,
                                          const f32x4_t (&acc)[D / 16], Out out) {
#pragma unroll
  for (int db = 0; db < D / 16; ++db)
    *reinterpret_cast<f32x4_t*>(tile + r * Block<D>::PITCH + 16 * db + 4 * g) = acc[db] * f;
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * D / 4; e += NW * 64) {
    const int row = e / (D / 4), c = e % (D / 4) * 4;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w)
      sum += *reinterpret_cast<const f32x4_t*>(lds + w * Block<D>::FLOATS + row * Block<D>::PITCH + c);
    out(row, c, sum);
  }
}

}  // namespace kl
