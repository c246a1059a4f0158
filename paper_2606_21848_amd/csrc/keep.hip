// The end of a draft step: the accepted rows of a drafted tree move up behind the
// rows that were cached before it (row n + path[k] to row n + k), so that the
// sequence lies whole again.
//
// One workgroup per (sequence, group) holds every moved row in registers between
// its reads and its writes, with a barrier between them: a path may name rows that
// are destinations too, in any order, and the same row twice. A pass reads and
// writes each accepted row once; what bounds it is one chain of memory latencies
// (kept count, path and table entries, rows): 2.2 us for 8 rows of one sequence, 3.8 us for
// 64 sequences of up to 64 rows in 8 groups of 128 (2.2 MB).

#include "kl_device.h"
#include "kl_internal.h"

namespace kl {
namespace {

constexpr int kThreads = 256;

template <int SLICES>  // 16-byte slices per row
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepParams p) {
  constexpr int PER = kMaxDrafts * SLICES / kThreads;  // slices per thread
  static_assert(kMaxDrafts * SLICES % kThreads == 0, "whole slices per thread");
  const int g = blockIdx.x % p.G, b = blockIdx.x / p.G;
  const int sl = threadIdx.x % SLICES, k0 = threadIdx.x / SLICES;
  const int kept = min(p.kept[b], p.T), n = p.lengths_before[b];
  const int cap = p.paged ? p.max_blocks << p.block_shift : p.L_max;
  // The cache row of position n + at, or -1 where there is none (sums in 64 bits:
  // a length is whatever the device holds).
  auto row_of = [&](int at) -> long {
    const long pos = (long)n + at;
    if (pos < 0 || pos >= cap) return -1;
    if (!p.paged) return ((long)b * p.G + g) * p.L_max + pos;
    const int blk = p.table[(size_t)b * p.max_blocks + (pos >> p.block_shift)];
    if (blk < 0 || blk >= p.num_blocks) return -1;
    return (((long)blk * p.G + g) << p.block_shift) + (pos & ((1 << p.block_shift) - 1));
  };
  u32x4* data = static_cast<u32x4*>(p.data);
  u32x4 x[PER];
  long to[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int k = k0 + u * (kThreads / SLICES);
    to[u] = -1;
    if (k >= kept) continue;
    const int from = p.path[(size_t)b * p.T + k];
    if (from < 0 || from >= p.T || from == k) continue;
    const long src = row_of(from);
    if (src < 0) continue;
    to[u] = row_of(k);
    x[u] = data[src * SLICES + sl];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u)
    if (to[u] >= 0) data[to[u] * SLICES + sl] = x[u];
}

}  // namespace

hipError_t launch_keep(const KeepParams& p, hipStream_t st) {
  const dim3 grid((unsigned)p.B * p.G);
  switch (p.D * (p.dtype == KL_BF16 ? 2 : 4) / 16) {
    case 8: hipLaunchKernelGGL(keep_kernel<8>, grid, dim3(kThreads), 0, st, p); break;
    case 16: hipLaunchKernelGGL(keep_kernel<16>, grid, dim3(kThreads), 0, st, p); break;
    case 32: hipLaunchKernelGGL(keep_kernel<32>, grid, dim3(kThreads), 0, st, p); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace kl
