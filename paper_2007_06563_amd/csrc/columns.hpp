// Sums of the columns of float32 parts, in the parts' order: what kernels that sum over rows leave,
// a part a workgroup (or wave), becomes the sum in the output's type.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "narrow.hpp"

namespace hobflops {

// part: [parts][stride]; out[0][c] the sum of column c, out[1][c] that of column second + c, c < cols
// (either may be null). A workgroup has 64 columns; its waves take every sixteenth part each, and
// their sums meet in LDS.
template <class T>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* part, int64_t parts, int64_t stride,
                                                           int64_t cols, int64_t second,
                                                           typename T::elem* out0, typename T::elem* out1) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  typename T::elem* out = blockIdx.y ? out1 : out0;
  if (!out) return;
  const float* p = part + (blockIdx.y ? second : 0) + (c < cols ? c : 0);
  float v = 0.0f;
  int64_t i = wave;
  for (; i + 7 * 16 < parts; i += 8 * 16) {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = p[(i + 16 * j) * stride];
#pragma unroll
    for (int j = 0; j < 8; ++j) v += e[j];
  }
  for (; i < parts; i += 16) v += p[i * stride];
  sums[wave][lane] = v;
  __syncthreads();
  if (wave || c >= cols) return;
#pragma unroll
  for (int j = 1; j < 16; ++j) v += sums[j][lane];
  out[c] = (typename T::elem)v;
}

template <class T>
void launch_column_sums(const float* part, int64_t parts, int64_t stride, void* out0, void* out1, int64_t cols,
                        int64_t second, hipStream_t s) {
  column_sums_kernel<T><<<dim3((unsigned)((cols + 63) / 64), 2), 1024, 0, s>>>(
      part, parts, stride, cols, second, (typename T::elem*)out0, (typename T::elem*)out1);
}

}  // namespace hobflops
