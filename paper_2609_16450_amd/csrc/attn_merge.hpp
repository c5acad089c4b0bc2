// The kernel that merges the key-split partials of a bf16 attention launch.
#pragma once

#include "attn_common.hpp"

namespace eb {
namespace {

// Combine the key-split partials of each (block row, query head), one wavefront per pair.
template <int D, int kGroup>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnParams p, int total_block, int batch) {
  const int rh = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rh >= total_block * p.hq) return;  // uniform per wavefront
  attn_merge_pair<D, kGroup>(p, rh, batch, threadIdx.x & 63);
}

template <int D>
void launch_merge(const AttnParams& p, int total_block, int batch, hipStream_t s) {
  const long pairs = static_cast<long>(total_block) * p.hq;
  const dim3 grid(static_cast<unsigned>((pairs + 3) / 4));
  if (p.nsplit <= 4)
    hipLaunchKernelGGL((attn_merge_kernel<D, 4>), grid, dim3(256), 0, s, p, total_block, batch);
  else if (p.nsplit <= 8)
    hipLaunchKernelGGL((attn_merge_kernel<D, 8>), grid, dim3(256), 0, s, p, total_block, batch);
  else
    hipLaunchKernelGGL((attn_merge_kernel<D, 16>), grid, dim3(256), 0, s, p, total_block, batch);
}

}  // namespace
}  // namespace eb
