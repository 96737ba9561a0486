// The gated feed-forward block, h = act(x Wg^T) * (x Wu^T), and its gradients
// from 8-bit checkpoints:
//   dg = dh * u * act'(g), du = dh * act(g),
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x.
// Products run on the 16x16x32 matrix instruction with float32 sums. (32x32x16 needs fewer
// cycles but took longer: at these rates power sets the clock. 8192 x 22528 x 4096 with values of
// 0 runs in 0.92 ms, with normal ones in 1.10 ms.)
//
// Roundings to 16 bits: h once, from float32 products; dg, du and the values of x's blocks, as operands
// of the matrix instruction; dx and the weights' gradients once, from float32 sums. g and u in float32
// become 8-bit blocks directly.
//
// dg and du as one operand each: training steps are 0.0024 of their outputs' size off 64 bits in bfloat16,
// 0.0003 in float16, of which the outputs' own rounding is 0.0017 and 0.0002. Two operands each (the
// rounded value and what it leaves) would double the products, 1.1 ms of a step of 4096 x 4096 x 11264, which takes 1.8.
// In float16 dg and du also have its range; gradients are linear in dh, whose scale is the caller's.
//
// Every sum has a fixed order: results do not change between runs.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "gemm.hpp"
#include "narrow.hpp"
#include "tiles.hpp"

namespace hobflops {
namespace {

// ---- the products ------------------------------------------------------------

struct ForwardArgs {
  const void *w[2], *x;
  int64_t ldw, ldx, T_, F, K, ldh;
  void* h;
  GatedBlocks gate, up;
  int act;
  uint32_t ni, nj;
};

// The scale and codes of 32 rows of a column, from two tiles' sums: a group of token t from f0 on.
template <int kFmt>
__device__ __forceinline__ void store_block(const GatedBlocks& b, int64_t t, int64_t F, int64_t f0,
                                            int lane, bool ok, f32x4 v0, f32x4 v1) {
  const int q = lane >> 4;
  uint32_t a = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t m0 = f0 + 4 * q + r < F ? finite_abs(v0[r]) : 0u;
    const uint32_t m1 = f0 + 16 + 4 * q + r < F ? finite_abs(v1[r]) : 0u;
    a = a > m0 ? a : m0;
    a = a > m1 ? a : m1;
  }
  const auto x = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  a = x[0] > x[1] ? x[0] : x[1];
  const auto y = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  a = y[0] > y[1] ? y[0] : y[1];
  const int k = block_scale<kFmt>(a);
  const float s = pow2f(-k);
  uint32_t w[2] = {encode4<kFmt>(v0[0] * s, v0[1] * s, v0[2] * s, v0[3] * s),
                   encode4<kFmt>(v1[0] * s, v1[1] * s, v1[2] * s, v1[3] * s)};
  gather_rows(w[0], w[1]);
  if (!ok || f0 >= F) return;
  if (q == 0) b.scales[t * ((F + 31) / 32) + f0 / 32] = (uint8_t)(k + 127);
  const int64_t f = f0 + 8 * q;
  uint8_t* p = b.codes + t * F + f;
  if (f + 8 <= F) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (f + r < F) p[r] = (uint8_t)(w[r >> 2] >> (8 * (r & 3)));
  }
}

// h = act(x Wg^T) * (x Wu^T): the tile's rows are BI / 2 of w_gate and the same of w_up, a wave
// has both sums of its outputs.
template <class T, int kFmt, int BI, int BJ, int WI, int WJ, int S>
__device__ __forceinline__ void forward_tile(const ForwardArgs& p, uint8_t* const (&sa)[S],
                                             uint8_t* const (&sb)[S]) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int NW = WI * WJ, NI = BI / WI / 32, NJ = BJ / WJ / 16;  // NI of each projection
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t ti, tj;
  tile_of(blockIdx.x, p.ni, p.nj, ti, tj);
  const int64_t i0 = (int64_t)ti * (BI / 2), j0 = (int64_t)tj * BJ;
  LoadRows<BI, NW, 2> la;
  LoadRows<BJ, NW, 1> lb;
  const void* const xs[1] = {p.x};
  la.start(p.w, p.ldw, p.F, i0, p.K, 0, wave, lane);
  lb.start(xs, p.ldx, p.T_, j0, p.K, 0, wave, lane);
  const int wi = wave % WI, wj = wave / WI;
  ReadRows<T, 2 * NI, BI / 2> ra;
  ReadRows<T, NJ, 0> rb;
  ra.start(wi * NI * 16, lane);
  rb.start(wj * NJ * 16, lane);
  f32x4 acc[2 * NI][NJ] = {};
  const auto load = [&](int s) {
    la.load(sa[s], wave);
    lb.load(sb[s], wave);
  };
  sum_tiles<T, 2 * NI, NJ, (BI + BJ) / 8 / NW, S>(acc, sa, sb, ra, rb, load,
                                                  (int)((p.K + kStepK - 1) / kStepK));
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t t = j0 + wj * NJ * 16 + 16 * j + (lane & 15);
    const bool ok = t < p.T_;
    typename T::elem* row = (typename T::elem*)p.h + (ok ? t : 0) * p.ldh;
#pragma unroll
    for (int i = 0; i < NI; i += 2) {
      const int64_t f = i0 + wi * NI * 16 + 16 * i;
      f32x4 v[2];
#pragma unroll
      for (int r = 0; r < 8; ++r)
        v[r >> 2][r & 3] = gate_act(acc[i + (r >> 2)][j][r & 3], p.act) * acc[NI + i + (r >> 2)][j][r & 3];
      store_rows<T>(row + f, p.F - f, ok, lane, v[0], v[1]);
      if constexpr (kFmt >= 0) {
        store_block<kFmt>(p.gate, t, p.F, f, lane, ok, acc[i][j], acc[i + 1][j]);
        store_block<kFmt>(p.up, t, p.F, f, lane, ok, acc[NI + i][j], acc[NI + i + 1][j]);
      }
    }
  }
#endif
}

// 256 x 256 sums a workgroup, 128 of each projection, one workgroup of eight waves on a CU. Bound by the matrix
// instructions, which are busy 73 % of the time: 8192 x 4096 x 11264 in 1.09 ms, 1.38 PFLOP/s, without any
// LDS bank conflict. (A library product of these sizes, without the activation: 0.95 ms.) With checkpoints 62 %:
// 4096 x 4096 x 11264 in 635 us, without 569; 1408 tiles are 5.5 rounds and take 6, and a
// tile's blocks are formed and stored with nothing beside them.
template <class T, int kFmt>
__global__ __launch_bounds__(512, 2) void forward_kernel(ForwardArgs p) {
  HOBFLOPS_STAGES2(256, 256);
  forward_tile<T, kFmt, 256, 256, 2, 4, 2>(p, sa, sb);
}
// 128 x 64 sums, where large tiles would be too few: two workgroups on a CU, three stages. Bound by the reads of the
// weights for few tokens (1 x 4096 x 11264: 39 us, 4.7 TB/s), by latency, of LDS too, in between
// (333 x 1000 x 2730: 18.0 us, of which 5 for the first and last step, 0.7 a step of 64 k).
template <class T, int kFmt>
__global__ __launch_bounds__(256, 2) void forward_small_kernel(ForwardArgs p) {
  HOBFLOPS_STAGES3(128, 64);
  forward_tile<T, kFmt, 128, 64, 2, 2, 3>(p, sa, sb);
}
// 64 x 64 sums, for weights of few rows; bound by latency. 64 x 1000 x 2730: 11 us with weights from HBM, 5.5 from L2.
template <class T, int kFmt>
__global__ __launch_bounds__(256, 3) void forward_few_kernel(ForwardArgs p) {
  HOBFLOPS_STAGES3(64, 64);
  forward_tile<T, kFmt, 64, 64, 1, 4, 3>(p, sa, sb);
}

// Workgroups of dx, as many as `parts`, then those of the weights' gradients: in one launch they fill each
// other's last rounds.
template <class T, int B, int WJ>
__device__ __forceinline__ void grad_tiles_of(const GradArgs& dx, const GradArgs& dw, uint32_t parts,
                                              uint8_t* const (&sa)[2], uint8_t* const (&sb)[2]) {
  if (blockIdx.x < parts) {
    const uint32_t tiles = dx.ni * dx.nj;
    grad_tile<T, false, 2, B, B, WJ, 2>(dx, sa, sb, blockIdx.x % tiles, blockIdx.x / tiles);
  } else {
    grad_tile<T, true, 2, B, B, WJ, 2>(dw, sa, sb, blockIdx.x - parts, 0);
  }
}
// 256 x 256 sums a workgroup: bound by the matrix instructions. 4096 x 4096 x 11264: both products, 1.5 TFLOP,
// in 1.13 ms, 1.34 PFLOP/s (the library's two products at these layouts: 1.30 ms).
template <class T>
__global__ __launch_bounds__(512, 2) void grad_kernel(GradArgs dx, GradArgs dw, uint32_t parts) {
  HOBFLOPS_STAGES2(256, 256);
  grad_tiles_of<T, 256, 4>(dx, dw, parts, sa, sb);
}
// 128 x 128 sums, two workgroups on a CU: for what would be a few rounds of large tiles, or less than one.
// 3000 x 2048 x 5632: both products in 258 us, 1.07 PFLOP/s; 77 x 512 x 1408: 9.2 us, latency.
template <class T>
__global__ __launch_bounds__(256, 2) void grad_small_kernel(GradArgs dx, GradArgs dw, uint32_t parts) {
  HOBFLOPS_STAGES2(128, 128);
  grad_tiles_of<T, 128, 2>(dx, dw, parts, sa, sb);
}

// Up to eight codes, `left` of them.
__device__ __forceinline__ void load_codes(const uint8_t* p, int64_t left, uint32_t (&w)[2]) {
  if (left >= 8) {
    __builtin_memcpy(w, p, 8);
  } else {
    w[0] = w[1] = 0;
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < left) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
  }
}

// dg and du, rows [t][2 Fp] (du from Fp on, zeros from F to Fp), from dh and the blocks of g and u:
// 8 values a thread.
struct GateGradArgs {
  const void* dh;
  GatedBlocks gate, up;
  void* out;
  int64_t T_, F, Fp, ldh;
  int act;
};
template <class T, int kFmt>
__device__ __forceinline__ void gate_grad_of(const GateGradArgs& p, int64_t i, int64_t stride) {
  typedef typename T::elem E;
  const int64_t per = p.Fp / 8, n = p.T_ * per, groups = (p.F + 31) / 32;
  for (; i < n; i += stride) {
    const int64_t row = i / per, col = (i - row * per) * 8;
    typename T::vec8 dg, du;
    if (col < p.F) {
      const E* dh = (const E*)p.dh + row * p.ldh + col;
      const uint8_t *gc = p.gate.codes + row * p.F + col, *uc = p.up.codes + row * p.F + col;
      uint32_t wg[2], wu[2];
      typename T::vec8 d;
      if (col + 8 <= p.F) {
        __builtin_memcpy(&d, dh, 16);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = col + j < p.F ? dh[j] : (E)0.0f;
      }
      load_codes(gc, p.F - col, wg);
      load_codes(uc, p.F - col, wu);
      const int64_t s = row * groups + col / 32;
      const float sg = load_scale(p.gate.scales, s, HOBFLOPS_SCALE_POW2);
      const float su = load_scale(p.up.scales, s, HOBFLOPS_SCALE_POW2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 g = decode4<kFmt>(wg[h]), u = decode4<kFmt>(wu[h]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float a, da;
          gate_act_grad(g[j] * sg, p.act, a, da);
          const bool in = col + 4 * h + j < p.F;
          const float v = (float)d[4 * h + j];
          dg[4 * h + j] = in ? (E)(v * (u[j] * su) * da) : (E)0.0f;
          du[4 * h + j] = in ? (E)(v * a) : (E)0.0f;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) dg[j] = du[j] = (E)0.0f;
    }
    E* out = (E*)p.out + row * 2 * p.Fp + col;
    *(typename T::vec8*)out = dg;
    *(typename T::vec8*)(out + p.Fp) = du;
  }
}

// A code times its scale as an operand of the type. What blocks of x stand for is one of its values, but that x near
// the type's top may have been rounded up to 2^16 (2^128), where float16 ends at 65504 (bfloat16 at
// 255 * 2^120) and has infinity: the largest value, within the type's rounding, is taken for it. What is larger
// (only blocks of another type's values are) and what is not finite go where the type's rounding takes them.
template <class T>
__device__ __forceinline__ typename T::elem operand_of(float d, float s) {
  const float half = d * (0.5f * s);  // (2^128 is beyond float32)
  if (__builtin_fabsf(half) == 0.5f * T::kMax + 0.5f * T::kStep)
    return (typename T::elem)__builtin_copysignf(T::kMax, half);
  return round_product<T>(d, s);
}

// Rows [t][ldd] of the values of blocks, zeros from cols on: 8 a thread.
struct UnpackArgs {
  GatedBlocks blocks;
  void* out;
  int64_t rows, cols, ldd;
};
template <class T, int kFmt>
__device__ __forceinline__ void unpack_of(const UnpackArgs& p, int64_t i, int64_t stride) {
  typedef typename T::elem E;
  const int64_t per = p.ldd / 8, n = p.rows * per, groups = (p.cols + 31) / 32;
  for (; i < n; i += stride) {
    const int64_t row = i / per, col = (i - row * per) * 8;
    uint32_t w[2];
    load_codes(p.blocks.codes + row * p.cols + col, p.cols - col, w);
    const float s = load_scale(p.blocks.scales, row * groups + col / 32, HOBFLOPS_SCALE_POW2);
    typename T::vec8 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 d = decode4<kFmt>(w[h]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[4 * h + j] = col + 4 * h + j < p.cols ? operand_of<T>(d[j], s) : (E)0.0f;
    }
    *(typename T::vec8*)((E*)p.out + row * p.ldd + col) = v;
  }
}

// What the gradients' products read, in one launch. Bound by HBM: 4096 x 4096 x 11264 reads 208 and
// writes 218 MB (by the counters) in 73 us. (Forming dg and du where the products load them would do that once for every
// 256 columns, and their tiles go into LDS past the registers.) With a launch for each of the three, a short step's took 3 us more. The first workgroups write dg and du, the next the values of
// x, the last the weights' rows if they must be aligned.
template <class T, int kFmt>
__global__ __launch_bounds__(256) void prepare_kernel(GateGradArgs gate, UnpackArgs x, AlignArgs w, uint32_t gates,
                                                      uint32_t xs) {
  const uint32_t b = blockIdx.x;
  if (b < gates)
    gate_grad_of<T, kFmt>(gate, (int64_t)b * 256 + threadIdx.x, (int64_t)gates * 256);
  else if (b < gates + xs)
    unpack_of<T, kFmt>(x, (int64_t)(b - gates) * 256 + threadIdx.x, (int64_t)xs * 256);
  else
    align_rows_of<T>(w, (int64_t)(b - gates - xs) * 256 + threadIdx.x, (int64_t)(gridDim.x - gates - xs) * 256);
}

__global__ void zero_kernel(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * blockDim.x)
    p[i] = 0;
}

// What a call keeps in its workspace, by byte offsets; -1: not needed.
struct ForwardPlan {
  int64_t x = -1, wg = -1, wu = -1, bytes = 0;
};
ForwardPlan plan_forward(const hobflops_gated_desc& d) {
  ForwardPlan p;
  const int64_t Dp = round_up(d.D, 8);
  const bool rows = d.align >= 16 && d.D % 8 == 0;
  if (!rows || d.ldx % 8 != 0 || d.ldx >= (int64_t)1 << 21) p.x = take(&p.bytes, d.T * Dp * 2);
  if (!rows || d.ldw % 8 != 0 || d.ldw >= (int64_t)1 << 21) {
    p.wg = take(&p.bytes, d.F * Dp * 2);
    p.wu = take(&p.bytes, d.F * Dp * 2);
  }
  return p;
}

// The tiles of a gradient's product and the parts of its sum, by an estimate of their time in microseconds:
// rounds of workgroups (of 256 x 256 tiles one on a CU, of 128 x 128 two), each its steps of 64 k and about
// five more to start and end, at 1.42 and 0.8 a step; the parts of a sum are written and read once
// more in float32, 4 TB/s, and joined in a launch. Measured, us: dx 1000 x 4096, sums of 22528, in
// one part 222 (128 x 128), in parts 180 (256 x 256); 333 x 4096, in 128 x 128: one part 118, parts 97;
// 3000 x 2048, sums of 11264: 128 x 128 one on a CU 183, two 138; dW of 1000 x 4096 x 22528: 256 x 256 172,
// 128 x 128 191, of 1 x 512 x 2816 7.5 and 5.5. The weights' sum over T is never in parts: of small weights a
// few workgroups walk all of it, and a backward pass of 8192 x 256 x 512 takes 85 us, of 8192 x 512 x 1408 119.
struct Tiling {
  bool small;
  int splits;
};
constexpr int kMaxSplits = 32;
Tiling plan_tiles(int64_t rows, int64_t cols, int64_t K, bool may_split) {
  const int64_t steps = (K + kStepK - 1) / kStepK;
  Tiling best{false, 1};
  double least = -1.0;
  for (int small = 0; small < 2; ++small) {
    const int64_t side = small ? 128 : 256, slots = small ? 2 * kCUs : kCUs;
    const int64_t tiles = ((rows + side - 1) / side) * ((cols + side - 1) / side);
    const double step = small ? 0.8 : 1.42;
    for (int n = 1; n <= (may_split ? kMaxSplits : 1) && (n == 1 || steps / n >= 6); ++n) {
      const double rounds = (double)((tiles * n + slots - 1) / slots);
      double us = rounds * ((double)((steps + n - 1) / n) + 5.0) * step;
      if (n > 1) us += 4.0 + (double)(n + 1) * rows * cols * 4.0 / 4e6;
      if (least < 0.0 || us < least) {
        least = us;
        best = Tiling{small != 0, n};
      }
    }
  }
  return best;
}
struct BackwardPlan {
  int64_t x = -1, wg = -1, wu = -1, dgu = -1, part = -1, bytes = 0;
  int64_t Dp, Fp;
  Tiling dx, dw;
};
BackwardPlan plan_backward(const hobflops_gated_desc& d) {
  BackwardPlan p;
  p.Dp = round_up(d.D, 8);
  p.Fp = round_up(d.F, kStepK);
  if (d.T == 0) return p;
  p.x = take(&p.bytes, d.T * p.Dp * 2);
  p.dgu = take(&p.bytes, d.T * 2 * p.Fp * 2);
  if (d.align < 16 || d.D % 8 != 0 || d.ldw % 8 != 0 || d.ldw >= (int64_t)1 << 21) {
    p.wg = take(&p.bytes, d.F * p.Dp * 2);
    p.wu = take(&p.bytes, d.F * p.Dp * 2);
  }
  p.dx = plan_tiles(d.T, d.D, 2 * p.Fp, true);
  p.dw = plan_tiles(2 * p.Fp, d.D, d.T, false);
  if (p.dx.splits > 1) p.part = take(&p.bytes, p.dx.splits * d.T * round_up(d.D, 4) * 4);
  return p;
}

template <class T, int kFmt>
void forward_tiles(ForwardArgs& p, hipStream_t s) {
  // Large tiles where there are about as many as 160: with 176 (512, or 333, x 4096 x 11264) 105 and 100 us against the
  // small ones' 141 and 111, with 88 (1 x 4096 x 11264) 89 against 44. The smallest where small ones leave half of the
  // CUs without one: with 88 of them (1 x 2048 x 5632) 17.0 us against 19.0, with 176 (128 x 2048 x 5632) 22.4
  // against 20.3. The rule does not look at T or K: few tokens of more than 20352 rows go to the large tiles as
  // well, 1 x 4096 x 20480 in 103 us where 20352 rows take 71 in the small ones, and few tiles walk a long K alone,
  // 1 x 8192 x 512 in 28 us.
  const int64_t big = ((p.F + 127) / 128) * ((p.T_ + 255) / 256);
  const int64_t small = ((p.F + 63) / 64) * ((p.T_ + 63) / 64);
  if (big >= 160) {
    p.ni = (uint32_t)((p.F + 127) / 128);
    p.nj = (uint32_t)((p.T_ + 255) / 256);
    forward_kernel<T, kFmt><<<p.ni * p.nj, 512, 0, s>>>(p);
  } else if (small > kCUs / 2) {
    p.ni = (uint32_t)((p.F + 63) / 64);
    p.nj = (uint32_t)((p.T_ + 63) / 64);
    forward_small_kernel<T, kFmt><<<p.ni * p.nj, 256, 0, s>>>(p);
  } else {
    p.ni = (uint32_t)((p.F + 31) / 32);
    p.nj = (uint32_t)((p.T_ + 63) / 64);
    forward_few_kernel<T, kFmt><<<p.ni * p.nj, 256, 0, s>>>(p);
  }
}

template <class T>
hipError_t forward(const hobflops_gated_desc& d, const GatedForward& c, int fmt, hipStream_t s) {
  const ForwardPlan plan = plan_forward(d);
  uint8_t* ws = (uint8_t*)c.workspace;
  const int64_t Dp = round_up(d.D, 8);
  ForwardArgs p{};
  p.x = c.x;
  p.w[0] = c.w_gate;
  p.w[1] = c.w_up;
  p.ldx = d.ldx;
  p.ldw = d.ldw;
  p.K = d.D;
  AlignArgs align{};
  align.cols = d.D;
  align.ldd = Dp;
  if (plan.x >= 0) {
    p.x = ws + plan.x;
    p.ldx = p.K = Dp;
    add_rows(align, 0, c.x, d.ldx, d.T, ws + plan.x);
  }
  if (plan.wg >= 0) {
    p.w[0] = ws + plan.wg;
    p.w[1] = ws + plan.wu;
    p.ldw = p.K = Dp;
    add_rows(align, 1, c.w_gate, d.ldw, d.F, ws + plan.wg);
    add_rows(align, 2, c.w_up, d.ldw, d.F, ws + plan.wu);
  }
  align_rows<T>(align, s);
  p.T_ = d.T;
  p.F = d.F;
  p.ldh = d.ldh;
  p.h = c.h;
  p.gate = c.gate;
  p.up = c.up;
  p.act = d.act;
  if (fmt == kE4M3)
    forward_tiles<T, kE4M3>(p, s);
  else if (fmt == kE5M2)
    forward_tiles<T, kE5M2>(p, s);
  else
    forward_tiles<T, -1>(p, s);
  return hipGetLastError();
}

// The tiles of a product, in p.ni and p.nj; their number.
uint32_t count_tiles(GradArgs& p, bool small) {
  const int64_t b = small ? 128 : 256;
  p.ni = (uint32_t)((p.ni_ + b - 1) / b);
  p.nj = (uint32_t)((p.nj_ + b - 1) / b);
  return p.ni * p.nj;
}
// dx in `parts` workgroups and dw in `tiles`, either may be none.
template <class T>
void grad_products(const GradArgs& dx, uint32_t parts, const GradArgs& dw, uint32_t tiles, bool small,
                   hipStream_t s) {
  if (small)
    grad_small_kernel<T><<<parts + tiles, 256, 0, s>>>(dx, dw, parts);
  else
    grad_kernel<T><<<parts + tiles, 512, 0, s>>>(dx, dw, parts);
}

template <class T>
hipError_t backward(const hobflops_gated_desc& d, const GatedBackward& c, int fmt, hipStream_t s) {
  typedef typename T::elem E;
  if (d.T == 0) {
    zero_kernel<<<1024, 256, 0, s>>>((uint16_t*)c.dw_gate, d.F * d.D);
    zero_kernel<<<1024, 256, 0, s>>>((uint16_t*)c.dw_up, d.F * d.D);
    return hipGetLastError();
  }
  const BackwardPlan plan = plan_backward(d);
  uint8_t* ws = (uint8_t*)c.workspace;
  const GateGradArgs gate{c.dh, c.gate, c.up, ws + plan.dgu, d.T, d.F, plan.Fp, d.ldh, d.act};
  const UnpackArgs x{c.x, ws + plan.x, d.T, d.D, plan.Dp};
  AlignArgs align{};
  if (plan.wg >= 0) {
    align.cols = d.D;
    align.ldd = plan.Dp;
    add_rows(align, 0, c.w_gate, d.ldw, d.F, ws + plan.wg);
    add_rows(align, 1, c.w_up, d.ldw, d.F, ws + plan.wu);
  }
  const unsigned gates = grid_of(d.T * plan.Fp / 8, 1 << 20), xs = grid_of(d.T * plan.Dp / 8, 65536);
  const unsigned grid = gates + xs + grid_of(align.rows[2] * align.ldd / 8, 65536);
  if (fmt == kE4M3)
    prepare_kernel<T, kE4M3><<<grid, 256, 0, s>>>(gate, x, align, gates, xs);
  else
    prepare_kernel<T, kE5M2><<<grid, 256, 0, s>>>(gate, x, align, gates, xs);
  GradArgs p{};
  p.F = d.F;
  p.Fp = plan.Fp;
  p.b = ws + plan.dgu;
  p.ldb = 2 * plan.Fp;
  p.ni_ = d.D;
  p.cols = plan.Dp;
  GradArgs w = p;
  w.a[0] = ws + plan.x;
  w.lda = plan.Dp;
  w.nj_ = w.bcols = 2 * plan.Fp;
  w.K = d.T;
  w.per = round_up(d.T, kStepK);
  w.out[0] = c.dw_gate;
  w.out[1] = c.dw_up;
  p.a[0] = c.w_gate;
  p.a[1] = c.w_up;
  p.lda = d.ldw;
  if (plan.wg >= 0) {
    p.a[0] = ws + plan.wg;
    p.a[1] = ws + plan.wu;
    p.lda = plan.Dp;
  }
  p.nj_ = d.T;
  p.K = 2 * plan.Fp;
  p.out[0] = c.dx;
  p.per = round_up((p.K + plan.dx.splits - 1) / plan.dx.splits, kStepK);
  const int splits = (int)((p.K + p.per - 1) / p.per);
  if (plan.part >= 0) p.part = (float*)(ws + plan.part);
  const uint32_t parts = count_tiles(p, plan.dx.small) * splits, tiles = count_tiles(w, plan.dw.small);
  if (plan.dx.small == plan.dw.small) {
    grad_products<T>(p, parts, w, tiles, plan.dx.small, s);
  } else {
    grad_products<T>(p, 0, w, tiles, plan.dw.small, s);
    grad_products<T>(p, parts, w, 0, plan.dx.small, s);
  }
  if (p.part)
    join_kernel<T><<<grid_of(d.T * round_up(d.D, 4) / 4, 4096), 256, 0, s>>>(p.part, splits, d.T,
                                                                             d.D, (E*)c.dx);
  return hipGetLastError();
}

}  // namespace

int64_t gated_forward_workspace(const hobflops_gated_desc& d) { return plan_forward(d).bytes; }
int64_t gated_backward_workspace(const hobflops_gated_desc& d) { return plan_backward(d).bytes; }

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
