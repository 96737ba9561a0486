// Sums of the columns of float32 parts, in the parts' order: what kernels that sum over rows leave,
// a part a workgroup (or wave), becomes the sum in the output's type. Short launches, bound by latency: 768 parts of 2 x 4096
// columns, 25 MB, 5.5 us.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "narrow.hpp"

namespace hobflops {

// The sums of up to 64 columns (as many as there are, `cols` or more) of part [parts][stride] by a workgroup of NW
// waves: each takes every NW-th part, their sums meet in LDS.
template <class T, int NW>
__device__ __forceinline__ void column_sum(const float* part, int64_t parts, int64_t stride, int64_t cols,
                                           typename T::elem* out) {
  __shared__ float sums[NW][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* p = part + (lane < cols ? lane : 0);
  float v = 0.0f;
  int64_t i = wave;
  for (; i + 7 * NW < parts; i += 8 * NW) {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = p[(i + NW * j) * stride];
#pragma unroll
    for (int j = 0; j < 8; ++j) v += e[j];
  }
  for (; i < parts; i += NW) v += p[i * stride];
  sums[wave][lane] = v;
  __syncthreads();
  if (wave || lane >= cols) return;
#pragma unroll
  for (int j = 1; j < NW; ++j) v += sums[j][lane];
  out[lane] = (typename T::elem)v;
}

// part: [parts][stride]; out0[c] the sum of column c, out1[c] that of column second + c, c < cols
// (either may be null).
template <class T>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* part, int64_t parts, int64_t stride,
                                                           int64_t cols, int64_t second,
                                                           typename T::elem* out0, typename T::elem* out1) {
  const int64_t c = (int64_t)blockIdx.x * 64;
  typename T::elem* out = blockIdx.y ? out1 : out0;
  if (out) column_sum<T, 16>(part + (blockIdx.y ? second : 0) + c, parts, stride, cols - c, out + c);
}

template <class T>
void launch_column_sums(const float* part, int64_t parts, int64_t stride, void* out0, void* out1, int64_t cols,
                        int64_t second, hipStream_t s) {
  column_sums_kernel<T><<<dim3((unsigned)((cols + 63) / 64), 2), 1024, 0, s>>>(
      part, parts, stride, cols, second, (typename T::elem*)out0, (typename T::elem*)out1);
}

}  // namespace hobflops
