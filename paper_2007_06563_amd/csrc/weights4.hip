// Products of a few tokens with 4-bit weights under group scales: y = x W^T,
// W[n][k] = code(n, k) * scale(n, k / group), and the gated form
// h = act(x Wg^T) * (x Wu^T).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

__device__ __forceinline__ float value4(uint32_t c) {
  const uint32_t m = c & 7u;
  const float v = m < 2 ? 0.5f * (float)m : pow2f((int)(m >> 1) - 1) * (m & 1u ? 1.5f : 1.0f);
  return __uint_as_float(__float_as_uint(v) | (c & 8u) << 28);
}

// One wave a row of W and token.
template <class T>
__global__ __launch_bounds__(256) void w4_kernel(W4Product p) {
  typedef typename T::elem E;
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y;
  if (n >= p.N) return;
  const int64_t groups = (p.K + p.group - 1) / p.group;
  float sum[2] = {0.0f, 0.0f};
  for (int w = 0; w < (p.w_up.codes ? 2 : 1); ++w) {
    const W4Matrix& m = w ? p.w_up : p.w;
    for (int64_t k = lane; k < p.K; k += 64) {
      const uint32_t c = m.codes[n * ((p.K + 1) / 2) + k / 2] >> (4 * (k & 1));
      sum[w] += (float)((const E*)p.x)[t * p.ldx + k] *
                (value4(c) * load_scale(m.scales, n * groups + k / p.group, p.scale));
    }
    for (int o = 32; o; o >>= 1) sum[w] += __shfl_xor(sum[w], o);
  }
  if (lane == 0)
    ((E*)p.y)[t * p.ldy + n] = (E)(p.w_up.codes ? gate_act(sum[0], p.act) * sum[1] : sum[0]);
}

}  // namespace

hipError_t launch_w4(const W4Product& p, hipStream_t stream) {
  if (p.T == 0) return hipSuccess;
  const dim3 grid((unsigned)((p.N + 3) / 4), (unsigned)p.T);
  if (p.type == HOBFLOPS_TYPE_BF16)
    w4_kernel<TypeBF16><<<grid, 256, 0, stream>>>(p);
  else
    w4_kernel<TypeF16><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace hobflops
