// Scored keyless attention and drafted-token decode, the plain form: 16 lanes per
// row, each holding D / 16 columns, one row of the other operand after another,
// fp32 arithmetic. Right for every case, and the yardstick of the tiled kernels.

#include <type_traits>

#include "kl_device.h"
#include "kl_internal.h"

namespace kl {
namespace {

template <typename T>
__device__ __forceinline__ float ld(const T* p, size_t i) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)p[i] << 16);
  else return p[i];
}
template <typename T>
__device__ __forceinline__ void st(T* p, size_t i, float v) {
  if constexpr (sizeof(T) == 2) p[i] = (T)f32_to_bf16(v);
  else p[i] = v;
}

constexpr int kRows = 16;  // rows per workgroup

// Row loads and dot products of one row's 16 lanes.
template <typename T, int D>
struct Row {
  static constexpr int E = D / 16;
  float x[E];
  __device__ __forceinline__ void load(const T* p, int c) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = ld(p, c * E + e);
  }
  __device__ __forceinline__ float dot(const Row& o) const {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(x[e], o.x[e], s);
    return group_sum<16>(s);
  }
};

// The score of a pair from its scaled dot product, and d score / d dot product.
__device__ __forceinline__ float score_of(float z, float cap, float slope, float dist, float& bend) {
  bend = 1.f;
  if (cap > 0.f) {
    const float t = tanhf(z / cap);
    bend = 1.f - t * t;
    z = cap * t;
  }
  return z - slope * dist;
}

__device__ __forceinline__ void seen_rows(const ScoredParams& p, int b, int i, int& lo, int& hi) {
  const size_t r = (size_t)b * p.N + i;
  lo = p.first ? max(p.first[r], 0) : 0;
  hi = p.last ? min(p.last[r], p.N) : (p.causal ? i + 1 : p.N);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void forward_kernel(ScoredParams p) {
  constexpr int E = D / 16;
  const int h = blockIdx.x % p.H;
  const long rest = blockIdx.x / p.H;
  const int tiles = (p.N + kRows - 1) / kRows;
  const int b = (int)(rest / tiles), c = threadIdx.x & 15;
  const int i = (int)(rest % tiles) * kRows + (threadIdx.x >> 4);
  if (i >= p.N) return;
  const int g = h / (p.H / p.G);
  const T* Q = static_cast<const T*>(p.q) + (((size_t)b * p.N + i) * p.H + h) * D;
  const T* V = static_cast<const T*>(p.v) + ((size_t)b * p.N * p.G + g) * D;
  const float slope = p.slopes ? p.slopes[h] : 0.f;
  Row<T, D> q, v;
  q.load(Q, c);
  float acc[E], m = -INFINITY, l = 0.f, bend;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  int lo, hi;
  seen_rows(p, b, i, lo, hi);
  for (int j = lo; j < hi; ++j) {
    v.load(V + (size_t)j * p.G * D, c);
    const float s = score_of(q.dot(v) * p.scale, p.cap, slope, fabsf((float)(i - j)), bend);
    const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
    const float a = expf(m - ms), w = expf(s - ms);
    l = fmaf(l, a, w);
    m = mn;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(w, v.x[e], acc[e] * a);
  }
  const float inv = lo < hi ? 1.f / l : 0.f;
  const size_t row = ((size_t)b * p.N + i) * p.H + h;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    st(static_cast<T*>(p.out), row * D + c * E + e, acc[e] * inv);
    if (p.out_f32) p.out_f32[row * D + c * E + e] = acc[e] * inv;
  }
  if (p.lse && c == 0) p.lse[((size_t)b * p.H + h) * p.N + i] = lo < hi ? m + logf(l) : -INFINITY;
}

// dQ~ and Dd = rowsum(P * dP), one query row per 16 lanes.
template <typename T, int D>
__global__ __launch_bounds__(256) void dq_kernel(ScoredParams p) {
  constexpr int E = D / 16;
  const int h = blockIdx.x % p.H;
  const long rest = blockIdx.x / p.H;
  const int tiles = (p.N + kRows - 1) / kRows;
  const int b = (int)(rest / tiles), c = threadIdx.x & 15;
  const int i = (int)(rest % tiles) * kRows + (threadIdx.x >> 4);
  if (i >= p.N) return;
  const int g = h / (p.H / p.G);
  const size_t row = ((size_t)b * p.N + i) * p.H + h, lrow = ((size_t)b * p.H + h) * p.N + i;
  const T* V = static_cast<const T*>(p.v) + ((size_t)b * p.N * p.G + g) * D;
  const float slope = p.slopes ? p.slopes[h] : 0.f, lse = p.lse[lrow];
  Row<T, D> q, v, go;
  q.load(static_cast<const T*>(p.q) + row * D, c);
  go.load(static_cast<const T*>(p.dout) + row * D, c);
  float acc[E], dd = 0.f, bend;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  int lo, hi;
  seen_rows(p, b, i, lo, hi);
  for (int j = lo; j < hi; ++j) {
    v.load(V + (size_t)j * p.G * D, c);
    const float s = score_of(q.dot(v) * p.scale, p.cap, slope, fabsf((float)(i - j)), bend);
    dd = fmaf(expf(s - lse), go.dot(v), dd);
  }
  if (c == 0) p.Dd[lrow] = dd;
  for (int j = lo; j < hi; ++j) {
    v.load(V + (size_t)j * p.G * D, c);
    const float s = score_of(q.dot(v) * p.scale, p.cap, slope, fabsf((float)(i - j)), bend);
    const float ds = expf(s - lse) * (go.dot(v) - dd) * bend * p.scale;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(ds, v.x[e], acc[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) st(static_cast<T*>(p.dq), row * D + c * E + e, acc[e]);
}

// dV, one value row per 16 lanes, every head of its group after another.
template <typename T, int D>
__global__ __launch_bounds__(256) void dv_kernel(ScoredParams p) {
  constexpr int E = D / 16;
  const int g = blockIdx.x % p.G, R = p.H / p.G;
  const long rest = blockIdx.x / p.G;
  const int tiles = (p.N + kRows - 1) / kRows;
  const int b = (int)(rest / tiles), c = threadIdx.x & 15;
  const int j = (int)(rest % tiles) * kRows + (threadIdx.x >> 4);
  if (j >= p.N) return;
  const size_t vrow = ((size_t)b * p.N + j) * p.G + g;
  Row<T, D> q, v, go;
  v.load(static_cast<const T*>(p.v) + vrow * D, c);
  float acc[E], bend;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int h = g * R; h < (g + 1) * R; ++h) {
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    for (int i = 0; i < p.N; ++i) {
      int lo, hi;
      seen_rows(p, b, i, lo, hi);
      if (j < lo || j >= hi) continue;
      const size_t row = ((size_t)b * p.N + i) * p.H + h, lrow = ((size_t)b * p.H + h) * p.N + i;
      q.load(static_cast<const T*>(p.q) + row * D, c);
      go.load(static_cast<const T*>(p.dout) + row * D, c);
      const float s = score_of(q.dot(v) * p.scale, p.cap, slope, fabsf((float)(i - j)), bend);
      const float w = expf(s - p.lse[lrow]);
      const float ds = w * (go.dot(v) - p.Dd[lrow]) * bend * p.scale;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(w, go.x[e], fmaf(ds, q.x[e], acc[e]));
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) st(static_cast<T*>(p.dv), vrow * D + c * E + e, acc[e]);
}

// Drafted tokens: one (token, head) per workgroup, its 16 lane groups sharing the
// cached rows, merged once.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_kernel(TreeParams p) {
  constexpr int E = D / 16;
  const int h = blockIdx.x % p.H, t = blockIdx.x / p.H % p.T, b = blockIdx.x / p.H / p.T;
  const int g = h / (p.H / p.G), c = threadIdx.x & 15, sub = threadIdx.x >> 4;
  const int cap_rows = p.paged ? p.max_blocks << p.block_shift : p.L_max;
  const int n = min(max(p.lengths[b], 0), cap_rows), end = min(n + p.T, cap_rows);
  auto word = [&](int u) -> uint64_t {
    const uint64_t all = p.T == 64 ? ~0ull : (1ull << p.T) - 1;
    return p.tree ? p.tree[(size_t)b * p.T + u] & all : (2ull << u) - 1;
  };
  auto depth = [&](int u) { return __popcll(word(u) & ~(1ull << u)); };
  const uint64_t sees = word(t);
  const int here = depth(t);
  const size_t row = ((size_t)b * p.T + t) * p.H + h;
  const float slope = p.slopes ? p.slopes[h] : 0.f;
  Row<T, D> q, v;
  q.load(static_cast<const T*>(p.q) + row * D, c);
  float acc[E], m = -INFINITY, l = 0.f, bend;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int j = sub; j < end; j += 16) {
    if (j >= n && !(sees >> (j - n) & 1)) continue;
    size_t r;
    if (p.paged) {
      const int blk = p.table[(size_t)b * p.max_blocks + (j >> p.block_shift)];
      if (blk < 0 || blk >= p.num_blocks) continue;
      r = (((size_t)blk * p.G + g) << p.block_shift) + (j & ((1 << p.block_shift) - 1));
    } else {
      r = ((size_t)b * p.G + g) * p.L_max + j;
    }
    v.load(static_cast<const T*>(p.data) + r * D, c);
    const int dist = j < n ? n + here - j : here - depth(j - n);
    const float s = score_of(q.dot(v) * p.scale, p.cap, slope, fabsf((float)dist), bend);
    const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
    const float a = expf(m - ms), w = expf(s - ms);
    l = fmaf(l, a, w);
    m = mn;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(w, v.x[e], acc[e] * a);
  }
  __shared__ float s_acc[16][D], s_ml[16][2];
#pragma unroll
  for (int e = 0; e < E; ++e) s_acc[sub][c * E + e] = acc[e];
  if (c == 0) {
    s_ml[sub][0] = m;
    s_ml[sub][1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float mm = -INFINITY, total = 0.f, o = 0.f;
  for (int k = 0; k < 16; ++k) mm = fmaxf(mm, s_ml[k][0]);
  const float ms = mm == -INFINITY ? 0.f : mm;
  for (int k = 0; k < 16; ++k) {
    const float f = expf(s_ml[k][0] - ms);
    total = fmaf(s_ml[k][1], f, total);
    o = fmaf(s_acc[k][threadIdx.x], f, o);
  }
  st(static_cast<T*>(p.out), row * D + threadIdx.x, total == 0.f ? 0.f : o / total);
}

template <class F>
hipError_t pick(kl_dtype dtype, int D, F f) {
  if (dtype == KL_BF16) D == 128 ? f(uint16_t{}, std::integral_constant<int, 128>{})
                                 : f(uint16_t{}, std::integral_constant<int, 64>{});
  else D == 128 ? f(float{}, std::integral_constant<int, 128>{})
                : f(float{}, std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scored_forward(const ScoredParams& p, hipStream_t stream) {
  if (p.dtype == KL_BF16) return launch_scored_forward_bf16(p, stream);
  const dim3 grid((unsigned)p.H * p.B * ((p.N + kRows - 1) / kRows));
  return pick(p.dtype, p.D, [&](auto t, auto d) {
    hipLaunchKernelGGL((forward_kernel<decltype(t), decltype(d)::value>), grid, dim3(256), 0, stream, p);
  });
}

hipError_t launch_scored_backward(const ScoredParams& p, hipStream_t stream) {
  if (p.dtype == KL_BF16) return launch_scored_backward_bf16(p, stream);
  const unsigned tiles = (unsigned)p.B * ((p.N + kRows - 1) / kRows);
  return pick(p.dtype, p.D, [&](auto t, auto d) {
    hipLaunchKernelGGL((dq_kernel<decltype(t), decltype(d)::value>), dim3(p.H * tiles), dim3(256), 0,
                       stream, p);
    hipLaunchKernelGGL((dv_kernel<decltype(t), decltype(d)::value>), dim3(p.G * tiles), dim3(256), 0,
                       stream, p);
  });
}

hipError_t launch_tree_decode(const TreeParams& p, hipStream_t stream) {
  if (p.dtype == KL_BF16) return launch_tree_decode_bf16(p, stream);
  return pick(p.dtype, p.D, [&](auto t, auto d) {
    hipLaunchKernelGGL((tree_kernel<decltype(t), decltype(d)::value>), dim3(p.H * p.T * p.B),
                       dim3(256), 0, stream, p);
  });
}

}  // namespace kl
