// The gated feed-forward block, h = act(x Wg^T) * (x Wu^T), and its gradients
// from 8-bit checkpoints:
//   dg = dh * u * act'(g), du = dh * act(g),
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x.
// Products run on the 16x16x32 matrix instruction with float32 sums.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

// ---- a product of any strides ----------------------------------------------

// C[m][n] = sum_k A(m, k) B(n, k), operands by their strides; a 64x64 tile of
// four waves (32x32 each), 32 of K at a time through LDS.
struct Operand {
  const void* p;
  int64_t row, k;  // strides in elements
};
constexpr int kTile = 64, kTileK = 32, kPad = 8;

template <class T, class Out>
__global__ __launch_bounds__(256) void product_kernel(Operand a, Operand b, Out* c, int64_t ldc,
                                                      int64_t M, int64_t N, int64_t K, int add) {
  typedef typename T::elem E;
  __shared__ E sa[kTile][kTileK + kPad], sb[kTile][kTileK + kPad];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
  f32x4 acc[2][2] = {};
  for (int64_t k0 = 0; k0 < K; k0 += kTileK) {
    for (int i = tid; i < kTile * kTileK; i += 256) {
      const int r = i / kTileK, k = i % kTileK;
      const bool ka = k0 + k < K;
      sa[r][k] = ka && m0 + r < M ? ((const E*)a.p)[(m0 + r) * a.row + (k0 + k) * a.k] : (E)0.0f;
      sb[r][k] = ka && n0 + r < N ? ((const E*)b.p)[(n0 + r) * b.row + (k0 + k) * b.k] : (E)0.0f;
    }
    __syncthreads();
    typename T::vec8 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *(const typename T::vec8*)&sa[wm + 16 * i + (lane & 15)][8 * (lane >> 4)];
      fb[i] = *(const typename T::vec8*)&sb[wn + 16 * i + (lane & 15)][8 * (lane >> 4)];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = T::mfma(fa[i], fb[j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + wm + 16 * i + 4 * (lane >> 4) + r;
        const int64_t n = n0 + wn + 16 * j + (lane & 15);
        if (m < M && n < N) {
          const float v = acc[i][j][r] + (add ? (float)c[m * ldc + n] : 0.0f);
          c[m * ldc + n] = (Out)v;
        }
      }
}

template <class T, class Out>
void product(Operand a, Operand b, Out* c, int64_t ldc, int64_t M, int64_t N, int64_t K, int add,
             hipStream_t stream) {
  const dim3 grid((unsigned)((M + kTile - 1) / kTile), (unsigned)((N + kTile - 1) / kTile));
  product_kernel<T, Out><<<grid, 256, 0, stream>>>(a, b, c, ldc, M, N, K, add);
}

// h, and the blocks of both projections: one thread a value, 32 lanes a group.
template <class T, int kFmt>
__global__ __launch_bounds__(256) void gate_kernel(const float* g, const float* u, void* h,
                                                   int64_t T_, int64_t F, int64_t ldh, int act,
                                                   GatedBlocks gb, GatedBlocks ub) {
  const int64_t groups = (F + 31) / 32;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / (groups * 32), col = i - row * groups * 32;
  if (row >= T_) return;
  const float vg = col < F ? g[row * F + col] : 0.0f, vu = col < F ? u[row * F + col] : 0.0f;
  if (col < F) ((typename T::elem*)h)[row * ldh + col] = (typename T::elem)(gate_act(vg, act) * vu);
  if (kFmt < 0) return;
  constexpr int kF = kFmt < 0 ? 0 : kFmt;
  for (int w = 0; w < 2; ++w) {
    const float v = w ? vu : vg;
    const GatedBlocks& b = w ? ub : gb;
    uint32_t a = finite_abs(v);
    for (int m = 1; m < 32; m <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)a, m);
      a = a > o ? a : o;
    }
    const int k = block_scale<kF>(a);
    if ((col & 31) == 0) b.scales[row * groups + col / 32] = (uint8_t)(k + 127);
    if (col < F) b.codes[row * F + col] = (uint8_t)encode4<kF>(v * pow2f(-k), 0.0f, 0.0f, 0.0f);
  }
}

// dg, du [T][F] and x [T][D] from the blocks.
template <class T, int kFmt>
__global__ __launch_bounds__(256) void gate_grad_kernel(const void* dh, int64_t ldh, int64_t T_,
                                                        int64_t F, int act, GatedBlocks gb,
                                                        GatedBlocks ub, void* dg, void* du) {
  typedef typename T::elem E;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / F, col = i - row * F, groups = (F + 31) / 32;
  if (row >= T_) return;
  const int64_t s = row * groups + col / 32;
  const float g = decode4<kFmt>(gb.codes[i])[0] * load_scale(gb.scales, s, HOBFLOPS_SCALE_POW2);
  const float u = decode4<kFmt>(ub.codes[i])[0] * load_scale(ub.scales, s, HOBFLOPS_SCALE_POW2);
  const float d = (float)((const E*)dh)[row * ldh + col];
  float a, da;
  gate_act_grad(g, act, a, da);
  ((E*)dg)[i] = (E)(d * u * da);
  ((E*)du)[i] = (E)(d * a);
}

__global__ void zero_kernel(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * blockDim.x)
    p[i] = 0;
}

template <class T>
__global__ __launch_bounds__(256) void round_kernel(const float* src, typename T::elem* dst,
                                                    int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) dst[i] = (typename T::elem)src[i];
}

template <class T>
hipError_t forward(const hobflops_gated_desc& d, const GatedForward& p, int fmt, hipStream_t s) {
  if (d.T == 0) return hipSuccess;
  float* g = (float*)p.workspace;
  float* u = g + d.T * d.F;
  const Operand x{p.x, d.ldx, 1};
  product<T>(x, Operand{p.w_gate, d.ldw, 1}, g, d.F, d.T, d.F, d.D, 0, s);
  product<T>(x, Operand{p.w_up, d.ldw, 1}, u, d.F, d.T, d.F, d.D, 0, s);
  const int64_t n = d.T * ((d.F + 31) / 32) * 32;
  const unsigned grid = (unsigned)((n + 255) / 256);
  if (fmt == kE4M3)
    gate_kernel<T, kE4M3><<<grid, 256, 0, s>>>(g, u, p.h, d.T, d.F, d.ldh, d.act, p.gate, p.up);
  else if (fmt == kE5M2)
    gate_kernel<T, kE5M2><<<grid, 256, 0, s>>>(g, u, p.h, d.T, d.F, d.ldh, d.act, p.gate, p.up);
  else
    gate_kernel<T, -1><<<grid, 256, 0, s>>>(g, u, p.h, d.T, d.F, d.ldh, d.act, p.gate, p.up);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const hobflops_gated_desc& d, const GatedBackward& p, int fmt, hipStream_t s) {
  typedef typename T::elem E;
  if (d.T == 0) {
    zero_kernel<<<1024, 256, 0, s>>>((uint16_t*)p.dw_gate, d.F * d.D);
    zero_kernel<<<1024, 256, 0, s>>>((uint16_t*)p.dw_up, d.F * d.D);
    return hipGetLastError();
  }
  float* sum = (float*)p.workspace;  // dx before its rounding
  E* dg = (E*)(sum + d.T * d.D);
  E* du = dg + d.T * d.F;
  E* x = du + d.T * d.F;
  BlockTensor t{x, d.type, d.T, d.D, d.D, p.x.codes, p.x.scales, 32, HOBFLOPS_SCALE_POW2};
  hipError_t e = launch_block_unpack(t, fmt, s);
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)((d.T * d.F + 255) / 256);
  if (fmt == kE4M3)
    gate_grad_kernel<T, kE4M3><<<grid, 256, 0, s>>>(p.dh, d.ldh, d.T, d.F, d.act, p.gate, p.up, dg, du);
  else
    gate_grad_kernel<T, kE5M2><<<grid, 256, 0, s>>>(p.dh, d.ldh, d.T, d.F, d.act, p.gate, p.up, dg, du);
  product<T>(Operand{dg, 1, d.F}, Operand{x, 1, d.D}, (E*)p.dw_gate, d.D, d.F, d.D, d.T, 0, s);
  product<T>(Operand{du, 1, d.F}, Operand{x, 1, d.D}, (E*)p.dw_up, d.D, d.F, d.D, d.T, 0, s);
  product<T>(Operand{dg, d.F, 1}, Operand{p.w_gate, 1, d.ldw}, sum, d.D, d.T, d.D, d.F, 0, s);
  product<T>(Operand{du, d.F, 1}, Operand{p.w_up, 1, d.ldw}, sum, d.D, d.T, d.D, d.F, 1, s);
  const int64_t n = d.T * d.D;
  round_kernel<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(sum, (E*)p.dx, n);
  return hipGetLastError();
}

}  // namespace

int64_t gated_forward_workspace(const hobflops_gated_desc& d) { return 8 * d.T * d.F; }
int64_t gated_backward_workspace(const hobflops_gated_desc& d) {
  return 4 * d.T * d.D + 4 * d.T * d.F + 2 * d.T * d.D;
}

hipError_t launch_gated_forward(const hobflops_gated_desc& d, const GatedForward& p, int fmt,
                                hipStream_t stream) {
  return d.type == HOBFLOPS_TYPE_BF16 ? forward<TypeBF16>(d, p, fmt, stream)
                                      : forward<TypeF16>(d, p, fmt, stream);
}
hipError_t launch_gated_backward(const hobflops_gated_desc& d, const GatedBackward& p, int fmt,
                                 hipStream_t stream) {
  return d.type == HOBFLOPS_TYPE_BF16 ? backward<TypeBF16>(d, p, fmt, stream)
                                      : backward<TypeF16>(d, p, fmt, stream);
}

}  // namespace hobflops
