// Whole blocks of the paged K/V caches copied to other blocks (App. E keeps a
// stream's tokens in blocks wherever they lie: a fork that writes copies its
// last block, a compaction moves blocks to the front of the pool).
//
// A copy, bound by memory.  One workgroup copies up to 8 KB of one tensor of one
// pair: two 16-byte loads in flight per lane, past the caches both ways.
// Measured on one MI355X, 16,384 pairs drawn over a pool of 40,968 blocks of 2
// heads, d = 128, bf16 (537 MB read and written): 108 us (5.0 TB/s); with plain
// loads and stores 112; workgroups of 64, 128 or 512 threads, or 1,024 to 8,192
// workgroups that stride, 108 to 113.  (A plain copy of as many contiguous bytes
// takes 99.)
#include <hip/hip_runtime.h>

#include "../rotary.hpp"

namespace padoc {
namespace {

constexpr int kThreads = 256, kUnroll = 2;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Items: pieces of kThreads * kUnroll units, then the tensor, then the pair.
// SCALES: of 8-bit caches, whose scales the workgroup of K's first piece copies.
template <bool SCALES>
__global__ __launch_bounds__(kThreads) void copy_blocks_kernel(const CopyParams p, int64_t pieces, int64_t items) {
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t rest = item / pieces, piece = item - rest * pieces, pair = rest / 2;
    const int32_t from = p.pairs[2 * pair], to = p.pairs[2 * pair + 1];
    if (from < 0 || from >= p.src_blocks || to < 0 || to >= p.dst_blocks) continue;
    const u32x4* src = static_cast<const u32x4*>(rest % 2 ? p.v_src : p.k_src) + from * p.units;
    u32x4* dst = static_cast<u32x4*>(rest % 2 ? p.v_dst : p.k_dst) + to * p.units;
    const int64_t u0 = piece * (kThreads * kUnroll) + threadIdx.x;
    u32x4 x[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (u0 + i * kThreads < p.units) x[i] = __builtin_nontemporal_load(src + u0 + i * kThreads);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (u0 + i * kThreads < p.units) __builtin_nontemporal_store(x[i], dst + u0 + i * kThreads);
    if (SCALES && piece == 0 && rest % 2 == 0)
      for (int64_t u = threadIdx.x; u < p.s_units; u += kThreads)
        static_cast<u32x4*>(p.s_dst)[to * p.s_units + u] = static_cast<const u32x4*>(p.s_src)[from * p.s_units + u];
  }
}

}  // namespace

hipError_t launch_copy_blocks(const CopyParams& p, hipStream_t s) {
  if (p.n_pairs == 0) return hipSuccess;
  const int64_t pieces = (p.units + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  const int64_t items = p.n_pairs * 2 * pieces;
  const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20));
  if (p.s_units)
    hipLaunchKernelGGL(copy_blocks_kernel<true>, grid, dim3(kThreads), 0, s, p, pieces, items);
  else
    hipLaunchKernelGGL(copy_blocks_kernel<false>, grid, dim3(kThreads), 0, s, p, pieces, items);
  return hipGetLastError();
}

}  // namespace padoc
