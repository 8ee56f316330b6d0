// The last step of sums over rows (norm.hip, rms.hip): the workgroups' partial sums are added up.
#pragma once
#include "common.h"

namespace {

// Sums over rows from the workgroups' partial sums [groups][cols], of which the first `split` columns go to `first` and the others to `second`: 32
// columns a workgroup, 32 slices of the partial rows, added in a fixed order.  In 64 bits: 512 numbers added one after the other in 32
// would be most of the error of these sums, and the adds are not what the kernel waits for.  No rows (groups == 0): zeros.
__global__ __launch_bounds__(1024) void k_sum_parts(const float* __restrict__ partial, int32_t groups, int32_t cols, int32_t split,
                                                    float* __restrict__ first, float* __restrict__ second) {
  __shared__ double s[32][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
  double v = 0.;
  if (c < cols) {
    int k = slice;
    for (; k + 7 * 32 < groups; k += 8 * 32) {    // eight loads on their way at a time
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = partial[(int64_t)(k + j * 32) * cols + c];
#pragma unroll
      for (int j = 0; j < 8; ++j) v += (double)f[j];
    }
    for (; k < groups; k += 32) v += (double)partial[(int64_t)k * cols + c];
  }
  s[slice][col] = v;
  __syncthreads();
  if (threadIdx.x >= 32 || c >= cols) return;
  v = 0.;
#pragma unroll
  for (int k = 0; k < 32; ++k) v += s[k][col];
  (c < split ? first : second)[c < split ? c : c - split] = (float)v;
}

}  // namespace
