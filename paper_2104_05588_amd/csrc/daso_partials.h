// The sum of partial rows of two vectors' gradients, which workgroups leave in a workspace.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace daso {
namespace {

// dweight and dbias from the partial rows, in order: 16 columns a workgroup of 16 wavefronts, and 64
// shares of the rows with eight loads in flight each, which is all of them: 4 us for 512 rows of 2048 (with
// 16 shares 11).
__global__ __launch_bounds__(1024) void partials_kernel(const float* partial, int32_t count, int32_t d, float* dweight,
                                                        float* dbias) {
  __shared__ float shared[16][16];
  const int in = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int64_t c = blockIdx.x * 16 + in, width = 2 * int64_t(d);
  const float* const from = partial + min(c, width - 1);
  float sum = 0.0f;
  for (int32_t k = share; k < count; k += 512) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = from[min(k + 64 * i, count - 1) * width];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + 64 * i < count ? v[i] : 0.0f;
    sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if ((threadIdx.x & 63) < 16) shared[threadIdx.x >> 6][in] = sum;
  __syncthreads();
  if (threadIdx.x >= 16 || c >= width) return;
  sum = shared[0][in];
#pragma unroll
  for (int k = 1; k < 16; ++k) sum += shared[k][in];
  if (c < d) {
    if (dweight != nullptr) dweight[c] = sum;
  } else if (dbias != nullptr) {
    dbias[c - d] = sum;
  }
}

}  // namespace
}  // namespace daso
