// A linear layer with its epilogue, y = act(x W^T + b) + r, and its gradients:
//   z = x W^T + b,  dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum over rows of dz.
// Products run on the 16x16x32 matrix instruction with float32 sums, to which bias, activation and residual are
// applied before the one rounding of y. Few tokens read the weights once, straight to registers
// (direct_kernel); more go through LDS in tiles (gemm.hpp). Where tiles are too few for the chip, a sum is
// split and its parts are joined in their order in a second launch, which then has the epilogue.
//
// Roundings to 16 bits: y, dx, dW and db once each; z, kept for the backward pass, and dz as operand of
// both products. dz in one operand leaves gradients as far from 64 bits as their own rounding does
// again; two operands would double the products. db is summed from dz before it is rounded.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "columns.hpp"
#include "gemm.hpp"
#include "linear_plan.hpp"
#include "narrow.hpp"
#include "tiles.hpp"

namespace hobflops {
namespace {

// The activations for results of 16 bits: relative errors of some 2^-20, tails included, in about half of the
// instructions of gate_act (a tile's epilogue runs them with nothing beside: of 4096 x 4096 -> 11264, 369 us
// with a gelu of erfc).
// The normal distribution beyond |z|, over its density's exponential: exp(z^2 / 2) Phi(-|z|) as a polynomial of
// 1 / (1 + 0.35 |z|), fitted to a relative 3.2e-7 for |z| <= 14.5 (beyond it the product is below float32's range).
__device__ __forceinline__ float tail_ratio(float a) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.0f));
  float r = __builtin_fmaf(0.0489021204f, t, -0.201967299f);
  r = __builtin_fmaf(r, t, 0.240405872f);
  r = __builtin_fmaf(r, t, -0.0168311354f);
  r = __builtin_fmaf(r, t, 0.155871853f);
  r = __builtin_fmaf(r, t, 0.133378804f);
  r = __builtin_fmaf(r, t, 0.140267059f);
  return __builtin_fmaf(r, t, -2.71316530e-5f);
}
struct Gate {
  float p, e;  // the gate, and exp(-z^2 / 2)
};
// (The exponential instruction gives 0 below 2^-126: that is beyond |z| = 13.2, where z Phi(z) is below 2^-126 as well.)
__device__ __forceinline__ Gate gelu_gate(float z) {
  const float e = __builtin_amdgcn_exp2f(z * z * -0.721347520f), q = e * tail_ratio(__builtin_fabsf(z));
  return Gate{z < 0.0f ? q : 1.0f - q, e};
}
// exp(-|z|) 2^64, which the exponential instruction has down to |z| = 131, where z exp(z) is below bfloat16's range;
// within 2^-17.
__device__ __forceinline__ float far_exp(float z) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(__builtin_fabsf(z), -1.44269504f, 64.0f));
}
// sigmoid(z) and sigmoid(-z)
__device__ __forceinline__ Sigmoid silu_gate(float z) {
  const float e = far_exp(z) * 0x1p-64f, r = __builtin_amdgcn_rcpf(1.0f + e), far = e * r;
  return z < 0.0f ? Sigmoid{far, r} : Sigmoid{r, far};
}
// The activation of N values, or dy times its derivative. The choice of the activation stands around the values, so that they
// run through its chain of instructions beside each other. (A choice for each value: an epilogue of gelu, z and residual
// 20 us a round of tiles of 256 x 256, this 14.)
template <int N>
__device__ __forceinline__ void act_on(float (&v)[N], int act) {
  if (act == HOBFLOPS_GATE_SILU) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float z = v[k], e = far_exp(z), y = z * __builtin_amdgcn_rcpf(__builtin_fmaf(e, 0x1p-64f, 1.0f));
      v[k] = z < 0.0f ? y * e * 0x1p-64f : y;
    }
  } else if (act == HOBFLOPS_GATE_GELU) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] *= gelu_gate(v[k]).p;
  } else if (act == HOBFLOPS_GATE_RELU) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = v[k] > 0.0f || v[k] != v[k] ? v[k] : 0.0f;
  }
}
// A z that was kept as an infinity (float16 ends at 65504, the float32 z that y is of does not) has the slope of the
// largest float32, 0 or 1: infinity times the 0 of the gate's other half would be NaN.
__device__ __forceinline__ float finite_z(float z) {
  return __builtin_isinf(z) ? __builtin_copysignf(0x1.FFFFFEp127f, z) : z;
}
template <int N>
__device__ __forceinline__ void times_act_grad(float (&d)[N], const float (&kept)[N], int act) {
  if (act == HOBFLOPS_GATE_SILU) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float z = finite_z(kept[k]);
      const Sigmoid v = silu_gate(z);
      d[k] *= v.s * __builtin_fmaf(z, v.c, 1.0f);
    }
  } else if (act == HOBFLOPS_GATE_GELU) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float z = finite_z(kept[k]);
      const Gate v = gelu_gate(z);
      d[k] *= __builtin_fmaf(z, v.e * 0.398942280f, v.p);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] *= kept[k] > 0.0f ? 1.0f : kept[k] != kept[k] ? kept[k] : 0.0f;
  }
}

struct LinearArgs {
  const void *w, *x, *bias, *residual;
  void *y, *z;
  float* part;  // with splits: [splits][T][N rounded up to 4]
  int64_t ldw, ldx, ldr, ldy, T_, N, K, per;  // z: rows N apart; per: k of a split, a multiple of 64
  // (tiles through LDS: K without its last K % 8, which `tail` is)
  int act, tail;
  bool past;  // y and z go past the caches
  uint32_t ni, nj;
};

// Four values of a row from `col` on, zeros from `end` on.
template <class T>
__device__ __forceinline__ f32x4 load4(const typename T::elem* row, int64_t col, int64_t end) {
  typename T::elem e[4];
  if (col + 4 <= end) {
    __builtin_memcpy(e, row + col, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = col + i < end ? row[col + i] : (typename T::elem)0.0f;
  }
  return f32x4{(float)e[0], (float)e[1], (float)e[2], (float)e[3]};
}

#ifdef __HIP_DEVICE_COMPILE__
// Rows of a wave's sums in LDS: 16 tokens, NI * 16 values of each, and 16 bytes that keep the tokens on different banks.
template <int NI>
constexpr int kTileBytes = 16 * (NI * 64 + 16);

// What a wave wrote to LDS is read by its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The epilogue of a wave's sums, acc[i][j] of rows f0 + 16 i.. of W and tokens t0 + 16 j..: they go through LDS, 16
// tokens at a time, so that a lane has 8 neighbouring values of y and a token's lanes whole lines of y, z and the
// residual. The activation is applied in a loop of its own, whose code is there once for 16 tokens (unrolled
// over the whole tile it would not fit the instruction cache); the next 16 tokens' residual is under way meanwhile.
template <int NI>
constexpr int kPassesOf = NI / 2;  // of 16 tokens: 64 lanes with 8 values each
// The residual of 16 tokens from t0 on.
template <class T, int NI>
__device__ __forceinline__ void load_residual(const LinearArgs& p, int64_t f0, int64_t t0, int lane,
                                              typename T::vec8 (&r)[kPassesOf<NI>]) {
  typedef typename T::elem E;
  if (!p.residual || p.part) return;
  const int64_t f = f0 + 8 * (lane % (2 * NI));
#pragma unroll
  for (int n = 0; n < kPassesOf<NI>; ++n) {
    const int64_t t = t0 + n * (32 / NI) + lane / (2 * NI);
    const E* row = (const E*)p.residual + t * p.ldr;
    if (t >= p.T_) continue;
    if (f + 8 <= p.N) {
      __builtin_memcpy(&r[n], row + f, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (f + k < p.N) r[n][k] = row[f + k];
    }
  }
}

// more0: the residual of the first 16 tokens, loaded before the sums.
template <class T, int NI, int NJ>
__device__ __forceinline__ void store_tile(const LinearArgs& p, const f32x4 (&acc)[NI][NJ], int64_t f0, int64_t t0,
                                           uint8_t* lds, int lane, const typename T::vec8 (&more0)[kPassesOf<NI>]) {
  typedef typename T::elem E;
  typedef typename T::vec8 Vec;
  constexpr int kRow = NI * 64 + 16, kLanes = NI * 2, kAtOnce = 64 / kLanes, kPasses = kPassesOf<NI>;
  const int64_t f = f0 + 8 * (lane % kLanes);
  const int first = lane / kLanes;
  const bool whole = f + 8 <= p.N;
  uint8_t* const mine = lds + first * kRow + 32 * (lane % kLanes);
  const auto load8 = [&](const E* row) {
    Vec v = {};
    if (whole) {
      __builtin_memcpy(&v, row + f, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (f + k < p.N) v[k] = row[f + k];
    }
    return v;
  };
  const auto store8 = [&](E* row, const Vec& v) {
    if (whole) {
      store16(row + f, __builtin_bit_cast(u32x4v, v), p.past);
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (f + k < p.N) row[f + k] = v[k];
    }
  };
  float bias[8] = {};
  if (p.bias) {
    const Vec b = load8((const E*)p.bias);
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = (float)b[k];
  }
  const bool apart = p.act != kNoAct || p.z;  // bias, z and the activation in a loop before the residual's
  Vec more[2][kPasses] = {};
#pragma unroll
  for (int n = 0; n < kPasses; ++n) more[0][n] = more0[n];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      *(f32x4*)(lds + (lane & 15) * kRow + 64 * i + 16 * (lane >> 4)) = acc[i][j];
    if (j + 1 < NJ) load_residual<T, NI>(p, f0, t0 + 16 * (j + 1), lane, more[(j + 1) & 1]);
    wave_sync();
    if (apart) {
#pragma unroll 1
      for (int n = 0; n < kPasses; ++n) {
        f32x4* at = (f32x4*)(mine + n * kAtOnce * kRow);
        const f32x4 sum[2] = {at[0], at[1]};
        const int64_t t = t0 + 16 * j + n * kAtOnce + first;
        float v[8];
        Vec z;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[k] = sum[k >> 2][k & 3] + bias[k];
          z[k] = (E)v[k];
        }
        if (p.z && t < p.T_) store8((E*)p.z + t * p.N, z);
        act_on(v, p.act);
        at[0] = f32x4{v[0], v[1], v[2], v[3]};
        at[1] = f32x4{v[4], v[5], v[6], v[7]};
      }
    }
#pragma unroll
    for (int n = 0; n < kPasses; ++n) {
      const f32x4* at = (const f32x4*)(mine + n * kAtOnce * kRow);
      const f32x4 v[2] = {at[0], at[1]};
      const int64_t t = t0 + 16 * j + n * kAtOnce + first;
      Vec y;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float e = v[k >> 2][k & 3] + (apart ? 0.0f : bias[k]);
        y[k] = (E)(e + (float)more[j & 1][n][k]);
      }
      if (t < p.T_) store8((E*)p.y + t * p.ldy, y);
    }
    wave_sync();
  }
}
#endif

// A fragment of the last K % 8 values of 16 rows, and zeros: the lanes of the first 8 k have them.
template <class T>
__device__ __forceinline__ typename T::vec8 tail_of(const void* p, int64_t ld, int64_t rows, int64_t row0, int64_t K, int tail,
                                                    int lane) {
  u32x4v v = {0, 0, 0, 0};
  if (lane < 16) {
    const int64_t r = row0 + lane < rows ? row0 + lane : rows - 1;  // (sums of rows beyond the end: nobody stores them)
    const uint16_t* end = (const uint16_t*)p + r * ld + K + tail;
    if (K > 0) {
      __builtin_memcpy(&v, end - 8, 16);
      v = shifted_down(v, (uint32_t)(8 - tail) * 16);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < tail) v[j >> 1] |= (uint32_t)(end - tail)[j] << (16 * (j & 1));
    }
  }
  return __builtin_bit_cast(typename T::vec8, v);
}

template <class T, int BI, int BJ, int WI, int WJ, int S>
__device__ __forceinline__ void linear_tile(const LinearArgs& p, uint8_t* const (&sa)[S],
                                            uint8_t* const (&sb)[S]) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int NW = WI * WJ, NI = BI / WI / 16, NJ = BJ / WJ / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles = p.ni * p.nj, split = blockIdx.x / tiles;
  uint32_t ti, tj;
  tile_of(blockIdx.x - split * tiles, p.ni, p.nj, ti, tj);
  const int64_t i0 = (int64_t)ti * BI, j0 = (int64_t)tj * BJ;
  const int64_t k0 = (int64_t)split * p.per;
  const int64_t k1 = k0 + p.per < p.K ? k0 + p.per : p.K;
  LoadRows<BI, NW, 1> la;
  LoadRows<BJ, NW, 1> lb;
  const void *const ws[1] = {p.w}, *const xs[1] = {p.x};
  la.start(ws, p.ldw, p.N, i0, k1, k0, wave, lane);
  lb.start(xs, p.ldx, p.T_, j0, k1, k0, wave, lane);
  const int wi = wave % WI, wj = wave / WI;
  ReadRows<T, NI, 0> ra;
  ReadRows<T, NJ, 0> rb;
  ra.start(wi * NI * 16, lane);
  rb.start(wj * NJ * 16, lane);
  const int64_t f0 = i0 + wi * NI * 16, t0 = j0 + wj * NJ * 16;
  typename T::vec8 more[kPassesOf<NI>] = {};
  load_residual<T, NI>(p, f0, t0, lane, more);
  f32x4 acc[NI][NJ] = {};
  if (p.tail && split == 0) {
    typename T::vec8 b[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) b[j] = tail_of<T>(p.x, p.ldx, p.T_, t0 + 16 * j, p.K, p.tail, lane);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const typename T::vec8 a = tail_of<T>(p.w, p.ldw, p.N, f0 + 16 * i, p.K, p.tail, lane);
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = T::mfma(a, b[j], acc[i][j]);
    }
  }
  const auto load = [&](int s) {
    la.load(sa[s], wave);
    lb.load(sb[s], wave);
  };
  sum_tiles<T, NI, NJ, (BI + BJ) / 8 / NW, S>(acc, sa, sb, ra, rb, load,
                                              (int)((k1 - k0 + kStepK - 1) / kStepK));
  if (p.part) {
    const int64_t ldp = (p.N + 3) & ~(int64_t)3;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int64_t t = t0 + 16 * j + (lane & 15), at = f0 + 16 * i + 4 * (lane >> 4);
        if (t < p.T_ && at < p.N) *(f32x4*)(p.part + ((int64_t)split * p.T_ + t) * ldp + at) = acc[i][j];
      }
    return;
  }
  __syncthreads();  // the stages are free: no wave reads one or has a load into one under way
  // (two waves, or one, an array)
  constexpr int kEach = NW / 4;
  uint8_t* const stage = wave / kEach == 0 ? sa[0] : wave / kEach == 1 ? sa[1] : wave / kEach == 2 ? sb[0] : sb[1];
  store_tile<T, NI, NJ>(p, acc, f0, t0, stage + (wave % kEach) * kTileBytes<NI>, lane, more);
#endif
}

// 256 x 256 sums a workgroup, eight waves, one workgroup on a CU. Bound by the matrix instructions and the clock under them:
// 8192 x 11264 -> 4096 536 to 595 us from card to card (1.27 to 1.41 PFLOP/s; a library product 473 to 482), the
// instructions busy 75 % of the time; 4096 x 4096 -> 11264 with gelu, z and residual 327 to 345, 59 %: 704 tiles are 2.75 rounds
// that take 3, and a round's epilogue, 14 us, has nothing beside it.
template <class T>
__global__ __launch_bounds__(512, 2) void linear_kernel(LinearArgs p) {
  HOBFLOPS_STAGES2(256, 256);
  linear_tile<T, 256, 256, 2, 4, 2>(p, sa, sb);
}
// 128 x 128 sums, two workgroups on a CU (2048 x 4096 -> 4096: 60 us, in tiles of 256 x 256 84).
template <class T>
__global__ __launch_bounds__(256, 2) void linear_small_kernel(LinearArgs p) {
  HOBFLOPS_STAGES2(128, 128);
  linear_tile<T, 128, 128, 2, 2, 2>(p, sa, sb);
}
// Launches of about a workgroup a CU, which nothing else hides the latency of: four stages of 128 x 128 sums, six of 64 x
// 128 or eight of 64 x 64 under way, and two waves on a SIMD. (1024 x 4096 -> 4096: 34 us, of linear_small_kernel's 44; 512 x
// 4096 -> 4096: 24 in 64 x 128, 28 in 128 x 128, 41; 256 x 4096 -> 4096: 16 in 64 x 64, 20, 27, 40; 32 x 4096 -> 11264: 19 in 64 x
// 64, 23 in 64 x 128; four waves with four stages, a wave on a SIMD: 37 and 31.)
template <class T>
__global__ __launch_bounds__(512, 2) void linear_deep_kernel(LinearArgs p) {
  HOBFLOPS_STAGES4(128, 128);
  linear_tile<T, 128, 128, 2, 4, 4>(p, sa, sb);
}
template <class T>
__global__ __launch_bounds__(512, 2) void linear_deepest_kernel(LinearArgs p) {
  HOBFLOPS_STAGES6(64, 128);
  linear_tile<T, 64, 128, 2, 4, 6>(p, sa, sb);
}
template <class T>
__global__ __launch_bounds__(512, 2) void linear_least_kernel(LinearArgs p) {
  HOBFLOPS_STAGES8(64, 64);
  linear_tile<T, 64, 64, 2, 4, 8>(p, sa, sb);
}

// Four values of parts that are `stride` apart, added in their order; eight parts' loads under way.
__device__ __forceinline__ f32x4 sum_parts(const float* part, int64_t stride, int parts) {
  f32x4 v = *(const f32x4*)part;
  int s = 1;
  for (; s + 8 <= parts; s += 8) {
    f32x4 e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = *(const f32x4*)(part + (s + j) * stride);
#pragma unroll
    for (int j = 0; j < 8; ++j) v += e[j];
  }
  for (; s < parts; ++s) v += *(const f32x4*)(part + s * stride);
  return v;
}

// The parts of a sum in their order, then the epilogue: 4 values a thread.
template <class T>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs p, int splits) {
  typedef typename T::elem E;
  const int64_t ldp = (p.N + 3) & ~(int64_t)3, n = p.T_ * ldp;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
    f32x4 v = sum_parts(p.part + i, n, splits);
    const int64_t row = quotient(i, ldp), col = i - row * ldp;
    if (p.bias) v += load4<T>((const E*)p.bias, col, p.N);
    if (p.z) {
      const float e[4] = {v[0], v[1], v[2], v[3]};
      store4<T>((E*)p.z + row * p.N, col, p.N, e);
    }
    f32x4 r = {};
    if (p.residual) r = load4<T>((const E*)p.residual + row * p.ldr, col, p.N);
    float e[4] = {v[0], v[1], v[2], v[3]};
    act_on(e, p.act);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] += r[k];
    store4<T>((E*)p.y + row * p.ldy, col, p.N, e);
  }
}

// Few tokens or small layers, rows of any alignment: a workgroup has 16 NI rows of W and 16 NJ tokens, its waves
// every kDirectWaves-th 64 k of them, each by itself: U times 64 k are under way to its registers (eight lanes read a
// row's line of 128 bytes), go through its own part of LDS into the matrix instruction's order, and no wave
// waits for another before the end, where the waves' sums meet, are added in the waves' order and take the
// epilogue. (Loading the matrix instruction's order from memory, where neighbouring lanes have different rows, reads
// 45 bytes a nanosecond on a CU at most.)
// Bound by the weights from HBM where they are many, 1 x 11264 -> 4096 in 16 us (5.7 TB/s), and by latency where not: 333 x 2730
// -> 1000 13 us, 77 x 1022 -> 2731 10.
constexpr int kDirectWaves = 8;
#ifdef __HIP_DEVICE_COMPILE__
// The loads of N times 16 rows and 64 k: 8 rows each.
template <class T, int N>
struct DirectRows {
  const typename T::elem* row[2 * N];  // the lane's, at its k
  int k[2];                            // of loads 0, 2, .. and 1, 3, ..
  __device__ __forceinline__ void start(const void* p, int64_t ld, int64_t rows, int64_t row0, int lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) k[i] = 8 * ((lane & 7) ^ ((4 * i + (lane >> 4)) & 7));
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      // rows beyond the end: the last one again, whose sums nobody stores
      const int64_t r = row0 + 8 * i + (lane >> 3);
      row[i] = (const typename T::elem*)p + (r < rows ? r : rows - 1) * ld + k[i & 1];
    }
  }
  __device__ __forceinline__ void load(u32x4v (&v)[2 * N], int64_t k0) const {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) __builtin_memcpy(&v[i], row[i] + k0, 16);
  }
  // The last, fewer than 64 values of a row, from k0 to K, and zeros.
  __device__ __forceinline__ void load_end(u32x4v (&v)[2 * N], int64_t k0, int64_t K) const {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      const int over = (int)(k0 + k[i & 1] + 8 - K);  // values of the lane's 8 beyond the end
      if (K >= 8) {
        // the 8 values that end there
        __builtin_memcpy(&v[i], row[i] + k0 - (over > 0 ? over : 0), 16);
        if (over > 0) v[i] = shifted_down(v[i], over < 8 ? (uint32_t)over * 16 : 128);
      } else {
        v[i] = u32x4v{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < 8 - over) v[i][j >> 1] |= (uint32_t)((const uint16_t*)(row[i] + k0))[j] << (16 * (j & 1));
      }
    }
  }
};
#endif

template <class T, int NI, int NJ, int U>
__global__ __launch_bounds__(kDirectWaves * 64) void direct_kernel(LinearArgs p) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename T::elem E;
  typedef typename T::vec8 Vec;
  constexpr int kStage = (NI + NJ) * 2048, kSums = NI * NJ * 1024;
  __shared__ __align__(1024) uint8_t lds[kDirectWaves * (kStage > kSums ? kStage : kSums)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t ti, tj;
  tile_of(blockIdx.x, p.ni, p.nj, ti, tj);
  const int64_t f0 = (int64_t)ti * NI * 16, t0 = (int64_t)tj * NJ * 16;
  DirectRows<T, NI> la;
  DirectRows<T, NJ> lb;
  la.start(p.w, p.ldw, p.N, f0, lane);
  lb.start(p.x, p.ldx, p.T_, t0, lane);
  ReadRows<T, NI, 0> ra;
  ReadRows<T, NJ, 0> rb;
  ra.start(0, lane);
  rb.start(0, lane);
  uint8_t *const sa = lds + wave * kStage, *const sb = sa + NI * 2048;
  u32x4v a[U][2 * NI], b[U][2 * NJ];
  f32x4 acc[NI][NJ] = {};
  const auto write = [&](int u) {
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i) *(u32x4v*)(sa + i * 1024 + lane * 16) = a[u][i];
#pragma unroll
    for (int i = 0; i < 2 * NJ; ++i) *(u32x4v*)(sb + i * 1024 + lane * 16) = b[u][i];
    wave_sync();
  };
  const auto multiply = [&] {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      Vec fa[NI], fb[NJ];
#pragma unroll
      for (int i = 0; i < NI; ++i) fa[i] = ra.get(sa, i, ks);
#pragma unroll
      for (int j = 0; j < NJ; ++j) fb[j] = rb.get(sb, j, ks);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = T::mfma(fa[i], fb[j], acc[i][j]);
    }
    wave_sync();
  };
  // the wave's whole 64 k
  const int64_t whole = p.K / 64, mine = (whole - wave + kDirectWaves - 1) / kDirectWaves;
  if (mine > 0) {
    // (beyond the last the last one again, which nobody multiplies)
    const auto load = [&](int u, int64_t n) {
      const int64_t k = ((n < mine ? n : mine - 1) * kDirectWaves + wave) * 64;
      la.load(a[u], k);
      lb.load(b[u], k);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) load(u, u);
    int64_t n = 0;
    for (; n + U <= mine; n += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        write(u);
        load(u, n + U + u);
        multiply();
      }
    }
#pragma unroll
    for (int u = 0; u + 1 < U; ++u)
      if (n + u < mine) {
        write(u);
        multiply();
      }
  }
  if (p.K % 64 != 0 && wave == (int)(whole % kDirectWaves)) {
    la.load_end(a[0], whole * 64, p.K);
    lb.load_end(b[0], whole * 64, p.K);
    write(0);
    multiply();
  }
  __syncthreads();
  f32x4* const sums = (f32x4*)lds;  // [wave][NI * NJ][64]
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) sums[((wave * NI + i) * NJ + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int n = wave; n < NI * NJ; n += kDirectWaves) {
    // a lane has token t and four rows of W
    const int64_t at = f0 + 16 * (n / NJ) + 4 * (lane >> 4), t = t0 + 16 * (n % NJ) + (lane & 15);
    f32x4 v = sums[n * 64 + lane];
#pragma unroll
    for (int i = 1; i < kDirectWaves; ++i) v += sums[(i * NI * NJ + n) * 64 + lane];
    if (t >= p.T_ || at >= p.N) continue;
    if (p.bias) v += load4<T>((const E*)p.bias, at, p.N);
    if (p.z) {
      const float e[4] = {v[0], v[1], v[2], v[3]};
      store4<T>((E*)p.z + t * p.N, at, p.N, e);
    }
    f32x4 more = {};
    if (p.residual) more = load4<T>((const E*)p.residual + t * p.ldr, at, p.N);
    float e[4] = {v[0], v[1], v[2], v[3]};
    act_on(e, p.act);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] += more[k];
    store4<T>((E*)p.y + t * p.ldy, at, p.N, e);
  }
#endif
}

// ---- the gradients -----------------------------------------------------------

// dz in rows [t][ldo] (zeros from N to ldo) and the parts of db, with the alignment of x's and W's rows in the same
// launch: 256 columns and every `parts`-th 8 rows a workgroup, 8 values a thread. HBM-bound: 4096 x 11264, dy and z to dz, 52 to
// 58 us (5.3 to 4.8 TB/s).
struct DzArgs {
  const void *dy, *z;
  void* out;    // null: dy is read in place
  float* part;  // null: no db; else [parts][N rounded up to 8]
  int64_t T_, N, ldy, ldo;
  int act;
  uint32_t strips, parts;
};
template <class T>
__global__ __launch_bounds__(256) void linear_prepare_kernel(DzArgs p, AlignArgs rows) {
  typedef typename T::elem E;
  const uint32_t own = p.strips * p.parts;
  if (blockIdx.x >= own) {
    align_rows_of<T>(rows, (int64_t)(blockIdx.x - own) * 256 + threadIdx.x, (int64_t)(gridDim.x - own) * 256);
    return;
  }
  __shared__ float sums[8][256];
  const uint32_t strip = blockIdx.x % p.strips, part = blockIdx.x / p.strips;
  const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5;
  const int64_t col = (int64_t)strip * 256 + lane * 8;
  float db[8] = {};
  if (col < p.N) {
    for (int64_t t = (int64_t)part * 8 + sub; t < p.T_; t += (int64_t)p.parts * 8) {
      const E* dy = (const E*)p.dy + t * p.ldy + col;
      typename T::vec8 d = {}, z = {};
      if (col + 8 <= p.N) {
        __builtin_memcpy(&d, dy, 16);
        if (p.z) __builtin_memcpy(&z, (const E*)p.z + t * p.N + col, 16);
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (col + j < p.N) {
            d[j] = dy[j];
            if (p.z) z[j] = ((const E*)p.z)[t * p.N + col + j];
          }
      }
      float v[8], w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = (float)d[j];
        w[j] = (float)z[j];
      }
      if (p.z) times_act_grad(v, w, p.act);
      typename T::vec8 o;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        db[j] += v[j];
        o[j] = (E)v[j];
      }
      if (p.out) *(typename T::vec8*)((E*)p.out + t * p.ldo + col) = o;
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[sub][lane * 8 + j] = db[j];
  __syncthreads();
  const int64_t c = (int64_t)strip * 256 + threadIdx.x;
  float v = sums[0][threadIdx.x];
#pragma unroll
  for (int j = 1; j < 8; ++j) v += sums[j][threadIdx.x];
  if (c < p.N) p.part[(int64_t)part * ((p.N + 7) & ~(int64_t)7) + c] = v;
}

// Workgroups of dx, as many as `parts`, then those of dW: both products in one launch, so that dW's first tiles fill the
// CUs that dx's last ones leave. 4096 x 4096 -> 11264: 534 to 581 us from card to card (1.30 to 1.42 PFLOP/s), matrix instructions busy 79 %.
template <class T, int B, int WJ, int S>
__device__ __forceinline__ void linear_grad_tiles(const GradArgs& dx, const GradArgs& dw, uint32_t parts,
                                                  uint8_t* const (&sa)[S], uint8_t* const (&sb)[S]) {
  const bool first = blockIdx.x < parts;
  const uint32_t b = first ? blockIdx.x : blockIdx.x - parts;
  if (first)
    grad_tile<T, false, 1, B, B, WJ, S>(dx, sa, sb, b % (dx.ni * dx.nj), b / (dx.ni * dx.nj));
  else
    grad_tile<T, true, 1, B, B, WJ, S>(dw, sa, sb, b % (dw.ni * dw.nj), b / (dw.ni * dw.nj));
}
template <class T>
__global__ __launch_bounds__(512, 2) void linear_grad_kernel(GradArgs dx, GradArgs dw, uint32_t parts) {
  HOBFLOPS_STAGES2(256, 256);
  linear_grad_tiles<T, 256, 4>(dx, dw, parts, sa, sb);
}
template <class T>
__global__ __launch_bounds__(256, 2) void linear_grad_small_kernel(GradArgs dx, GradArgs dw, uint32_t parts) {
  HOBFLOPS_STAGES2(128, 128);
  linear_grad_tiles<T, 128, 2>(dx, dw, parts, sa, sb);
}
// As linear_deep_kernel: dx of 1024 x 4096 -> 4096 in 35 us, in tiles of two stages two a CU 44.
template <class T>
__global__ __launch_bounds__(512, 2) void linear_grad_deep_kernel(GradArgs dx, GradArgs dw, uint32_t parts) {
  HOBFLOPS_STAGES4(128, 128);
  linear_grad_tiles<T, 128, 4>(dx, dw, parts, sa, sb);
}

// What is left after the products, in one launch: the parts of dx and of dW joined in their order, 4 values a thread, and
// the parts of db, a column a thread's. (A launch each took a short step 3 us more.)
struct JoinArgs {
  const float* part;
  void* out;
  int64_t rows, cols;
  int splits;
  uint32_t groups;
};
template <class T>
__device__ __forceinline__ void join_of(const JoinArgs& p, int64_t i, int64_t stride) {
  const int64_t ldp = (p.cols + 3) & ~(int64_t)3, n = p.rows * ldp;
  for (i *= 4; i < n; i += stride * 4) {
    const f32x4 v = sum_parts(p.part + i, n, p.splits);
    const int64_t row = quotient(i, ldp), col = i - row * ldp;
    const float e[4] = {v[0], v[1], v[2], v[3]};
    store4<T>((typename T::elem*)p.out + row * p.cols, col, p.cols, e);
  }
}
template <class T>
__global__ __launch_bounds__(256) void linear_finish_kernel(JoinArgs dx, JoinArgs dw, const float* db_part, int64_t parts,
                                                            int64_t stride, int64_t cols, typename T::elem* db) {
  const uint32_t b = blockIdx.x;
  if (b < dx.groups) {
    join_of<T>(dx, (int64_t)b * 256 + threadIdx.x, (int64_t)dx.groups * 256);
  } else if (b < dx.groups + dw.groups) {
    join_of<T>(dw, (int64_t)(b - dx.groups) * 256 + threadIdx.x, (int64_t)dw.groups * 256);
  } else {
    const int64_t c = (int64_t)(b - dx.groups - dw.groups) * 64;
    column_sum<T, 4>(db_part + c, parts, stride, cols - c, db + c);
  }
}

template <class T>
__global__ __launch_bounds__(256) void zeros_kernel(typename T::elem* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    p[i] = (typename T::elem)0.0f;
}

// ---- launches ---------------------------------------------------------------

template <class T, int NI, int NJ, int U>
void launch_direct(LinearArgs& p, hipStream_t s) {
  p.ni = (uint32_t)((p.N + 16 * NI - 1) / (16 * NI));
  p.nj = (uint32_t)((p.T_ + 16 * NJ - 1) / (16 * NJ));
  direct_kernel<T, NI, NJ, U><<<p.ni * p.nj, kDirectWaves * 64, 0, s>>>(p);
}

template <class T>
hipError_t forward(const hobflops_linear_desc& d, const LinearForward& c, hipStream_t s) {
  LinearArgs p{};
  p.w = c.w;
  p.x = c.x;
  p.bias = c.bias;
  p.residual = c.residual;
  p.y = c.y;
  p.z = c.z;
  p.ldw = d.ldw;
  p.ldx = d.ldx;
  p.ldr = d.ldr;
  p.ldy = d.ldy;
  p.T_ = d.T;
  p.N = d.N;
  p.K = d.K;
  p.act = d.act;
  p.past = past_caches(d.T * d.N * 2);
  const ForwardPlan plan = plan_forward(d);
  if (plan.direct >= 0) {
    switch (plan.direct) {
      case 0: launch_direct<T, 1, 1, 4>(p, s); break;
      case 1: launch_direct<T, 1, 2, 4>(p, s); break;
      case 2: launch_direct<T, 1, 4, 2>(p, s); break;
      case 3: launch_direct<T, 2, 2, 3>(p, s); break;
      case 4: launch_direct<T, 2, 4, 2>(p, s); break;
      default: launch_direct<T, 4, 4, 1>(p, s);
    }
    return hipGetLastError();
  }
  uint8_t* ws = (uint8_t*)c.workspace;
  AlignArgs align{};
  align.cols = d.K;
  align.ldd = copied_ld(d.K);
  if (plan.x >= 0) {
    add_rows(align, 0, c.x, d.ldx, d.T, ws + plan.x);
    p.x = ws + plan.x;
    p.ldx = align.ldd;
  }
  if (plan.w >= 0) {
    add_rows(align, 1, c.w, d.ldw, d.N, ws + plan.w);
    p.w = ws + plan.w;
    p.ldw = align.ldd;
  }
  align_rows<T>(align, s);
  // (rows that were copied have zeros up to the multiple of 8)
  if (plan.x >= 0 && plan.w >= 0) p.K = round_up(d.K, 8);
  p.tail = (int)(p.K % 8);
  p.K -= p.tail;
  const int64_t splits = splits_of(p.K > 0 ? p.K : 1, plan.tiles.splits, &p.per);
  if (splits > 1) p.part = (float*)(ws + plan.part);
  const Kind& kind = kKinds[plan.tiles.kind];
  p.ni = (uint32_t)((d.N + kind.rows - 1) / kind.rows);
  p.nj = (uint32_t)((d.T + kind.cols - 1) / kind.cols);
  const unsigned grid = (unsigned)(p.ni * p.nj * splits);
  switch (plan.tiles.kind) {
    case 0: linear_kernel<T><<<grid, 512, 0, s>>>(p); break;
    case 1: linear_small_kernel<T><<<grid, 256, 0, s>>>(p); break;
    case 2: linear_deep_kernel<T><<<grid, 512, 0, s>>>(p); break;
    case 3: linear_deepest_kernel<T><<<grid, 512, 0, s>>>(p); break;
    default: linear_least_kernel<T><<<grid, 512, 0, s>>>(p);
  }
  if (p.part)
    linear_join_kernel<T><<<grid_of(d.T * round_up(d.N, 4) / 4, 4096), 256, 0, s>>>(p, (int)splits);
  return hipGetLastError();
}

uint32_t count_tiles(GradArgs& p, const Tiling& t) {
  const Kind& kind = kKinds[t.kind];
  p.ni = (uint32_t)((p.ni_ + kind.rows - 1) / kind.rows);
  p.nj = (uint32_t)((p.nj_ + kind.cols - 1) / kind.cols);
  return p.ni * p.nj;
}
template <class T>
void grad_products(const GradArgs& dx, uint32_t parts, const GradArgs& dw, uint32_t tiles, int kind, hipStream_t s) {
  if (parts + tiles == 0) return;
  switch (kind) {
    case 0: linear_grad_kernel<T><<<parts + tiles, 512, 0, s>>>(dx, dw, parts); break;
    case 1: linear_grad_small_kernel<T><<<parts + tiles, 256, 0, s>>>(dx, dw, parts); break;
    default: linear_grad_deep_kernel<T><<<parts + tiles, 512, 0, s>>>(dx, dw, parts);
  }
}

template <class T>
hipError_t backward(const hobflops_linear_desc& d, const LinearBackward& c, hipStream_t s) {
  typedef typename T::elem E;
  if (d.T == 0) {
    if (c.dw) zeros_kernel<T><<<1024, 256, 0, s>>>((E*)c.dw, d.N * d.K);
    if (c.db) zeros_kernel<T><<<16, 256, 0, s>>>((E*)c.db, d.N);
    return hipGetLastError();
  }
  const BackwardPlan plan = plan_backward(d, LinearNeed{c.dx != nullptr, c.dw != nullptr, c.db != nullptr});
  uint8_t* ws = (uint8_t*)c.workspace;
  DzArgs z{};
  z.dy = c.dy;
  z.z = d.act != kNoAct ? c.z : nullptr;
  z.out = plan.dz >= 0 ? ws + plan.dz : nullptr;
  z.part = plan.db >= 0 ? (float*)(ws + plan.db) : nullptr;
  z.T_ = d.T;
  z.N = d.N;
  z.ldy = d.ldy;
  z.ldo = plan.Np;
  z.act = d.act;
  z.strips = (uint32_t)((d.N + 255) / 256);
  z.parts = plan.parts;
  if (!z.out && !z.part) z.strips = z.parts = 0;
  AlignArgs align{};
  align.cols = d.K;
  align.ldd = plan.Kp;
  if (plan.x >= 0) add_rows(align, 0, c.x, d.ldx, d.T, ws + plan.x);
  if (plan.w >= 0) add_rows(align, 1, c.w, d.ldw, d.N, ws + plan.w);
  const unsigned grid = z.strips * z.parts + grid_of(align.rows[2] * align.ldd / 8, 65536);
  if (grid) linear_prepare_kernel<T><<<grid, 256, 0, s>>>(z, align);
  GradArgs p{};  // dx
  p.b = z.out ? z.out : c.dy;
  p.ldb = z.out ? plan.Np : d.ldy;
  p.ni_ = d.K;
  p.cols = plan.Kp;
  p.F = d.N;
  p.Fp = plan.Np;
  GradArgs w = p;
  w.a[0] = plan.x >= 0 ? ws + plan.x : c.x;
  w.lda = plan.x >= 0 ? plan.Kp : d.ldx;
  w.bcols = plan.Np;
  w.nj_ = d.N;
  w.K = d.T;
  w.out[0] = c.dw;
  p.a[0] = plan.w >= 0 ? ws + plan.w : c.w;
  p.lda = plan.w >= 0 ? plan.Kp : d.ldw;
  p.nj_ = d.T;
  p.K = plan.Np;
  p.out[0] = c.dx;
  const int64_t sx = splits_of(p.K, plan.dx.splits, &p.per), sw = splits_of(w.K, plan.dw.splits, &w.per);
  if (sx > 1) p.part = (float*)(ws + plan.part_x);
  if (sw > 1) w.part = (float*)(ws + plan.part_w);
  const uint32_t parts = c.dx ? count_tiles(p, plan.dx) * (uint32_t)sx : 0;
  const uint32_t tiles = c.dw ? count_tiles(w, plan.dw) * (uint32_t)sw : 0;
  if (plan.dx.kind == plan.dw.kind) {
    grad_products<T>(p, parts, w, tiles, plan.dx.kind, s);
  } else {
    grad_products<T>(p, 0, w, tiles, plan.dw.kind, s);
    grad_products<T>(p, parts, w, 0, plan.dx.kind, s);
  }
  JoinArgs jx{}, jw{};
  if (c.dx && p.part) jx = JoinArgs{p.part, c.dx, d.T, d.K, (int)sx, grid_of(d.T * round_up(d.K, 4) / 4, 4096)};
  if (c.dw && w.part) jw = JoinArgs{w.part, c.dw, d.N, d.K, (int)sw, grid_of(d.N * round_up(d.K, 4) / 4, 4096)};
  const unsigned last = jx.groups + jw.groups + (c.db ? (unsigned)((d.N + 63) / 64) : 0);
  if (last)
    linear_finish_kernel<T><<<last, 256, 0, s>>>(jx, jw, z.part, plan.parts, plan.Np, d.N, (E*)c.db);
  return hipGetLastError();
}

}  // namespace

int64_t linear_forward_workspace(const hobflops_linear_desc& d) { return plan_forward(d).bytes; }
int64_t linear_backward_workspace(const hobflops_linear_desc& d, const LinearNeed& need) {
  return plan_backward(d, need).bytes;
}

hipError_t launch_linear_forward(const hobflops_linear_desc& d, const LinearForward& p, hipStream_t s) {
  return d.type == HOBFLOPS_TYPE_BF16 ? forward<TypeBF16>(d, p, s) : forward<TypeF16>(d, p, s);
}
hipError_t launch_linear_backward(const hobflops_linear_desc& d, const LinearBackward& p, hipStream_t s) {
  return d.type == HOBFLOPS_TYPE_BF16 ? backward<TypeBF16>(d, p, s) : backward<TypeF16>(d, p, s);
}

}  // namespace hobflops
