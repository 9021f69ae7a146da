// Sums of partial results in an order that depends on their number alone: parameters' gradients of the sequence operators.
#ifndef SPRNN_SUMS_H_
#define SPRNN_SUMS_H_

#include "sprnn_seq.h"

namespace sprnn {

// put(i, sum over j < count of partial[j][i]) for i < width: 64 columns a workgroup, whose 16 wavefronts share out j.
template <typename Put>
__global__ __launch_bounds__(1024) void sum_partials_kernel(const float* partial, int count, int64_t width, Put put) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (i < width) {
    int j = wave;
    for (; j + 48 < count; j += 64) {
      const float p0 = partial[(int64_t)j * width + i], p1 = partial[(int64_t)(j + 16) * width + i];
      const float p2 = partial[(int64_t)(j + 32) * width + i], p3 = partial[(int64_t)(j + 48) * width + i];
      sum += (p0 + p1) + (p2 + p3);
    }
    for (; j < count; j += 16) sum += partial[(int64_t)j * width + i];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && i < width) {
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    put(i, sum);
  }
}

template <typename Put>
inline hipError_t launch_sum_partials(const float* partial, int count, int64_t width, const Put& put, hipStream_t stream) {
  return launch(sum_partials_kernel<Put>, dim3((unsigned)((width + 63) / 64)), dim3(1024), 0, stream, partial, count, width, put);
}

}  // namespace sprnn
#endif
