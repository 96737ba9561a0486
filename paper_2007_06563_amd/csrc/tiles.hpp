// What the matrix products around gemm.hpp's loop share: operands copied to aligned rows, a tile's sums to rows
// of memory, the tiles of gradients' products, and the joining of sums that were split.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gemm.hpp"
#include "narrow.hpp"

namespace hobflops {

constexpr int64_t kCUs = 256;

// a / b of numbers that are not negative, mostly below 2^32, where it takes a quarter of the instructions.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// Rows of operands as the products need them: 16-byte aligned, zeros from cols up to ldd. Up to three
// tensors of one width in a launch. (Whole chunks are read 16 bytes at a time whatever their alignment.)
struct AlignArgs {
  const void* src[3];
  void* dst[3];
  int64_t ld[3], rows[3];  // rows: of this tensor and those before
  int64_t cols, ldd;
};
// (i: the thread's number, of `stride` of them; so below)
template <class T>
__device__ __forceinline__ void align_rows_of(const AlignArgs& p, int64_t i, int64_t stride) {
  typedef typename T::elem E;
  const int64_t per = p.ldd / 8, n = p.rows[2] * per;
  for (; i < n; i += stride) {
    const int64_t all = quotient(i, per), col = (i - all * per) * 8;
    const int which = all < p.rows[0] ? 0 : all < p.rows[1] ? 1 : 2;
    const int64_t row = all - (which == 0 ? 0 : which == 1 ? p.rows[0] : p.rows[1]);
    const E* s = (const E*)p.src[which] + row * p.ld[which] + col;
    typename T::vec8 v = {};
    if (col + 8 <= p.cols) {
      __builtin_memcpy(&v, s, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (col + j < p.cols) v[j] = s[j];
    }
    *(typename T::vec8*)((E*)p.dst[which] + row * p.ldd + col) = v;
  }
}
template <class T>
__global__ __launch_bounds__(256) void align_kernel(AlignArgs p) {
  align_rows_of<T>(p, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

// Four values of a row, those before `end` of it.
template <class T>
__device__ __forceinline__ void store4(typename T::elem* p, int64_t col, int64_t end,
                                       const float (&v)[4]) {
  typedef typename T::elem E;
  if (col + 4 <= end) {
    E e[4] = {(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
    __builtin_memcpy(p + col, e, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < end) p[col + i] = (E)v[i];
  }
}

// A tile's sums stand with a lane's column lane % 16 and its rows 4 (lane / 16) + 0..3. For two tiles
// one after the other in rows, a word (of one value, or of several) of each, a and b, is exchanged
// between the four lanes of a column so that a lane has two neighbouring words: lane / 16 = q then
// holds words 2 q and 2 q + 1 of the column's eight.
__device__ __forceinline__ void gather_rows(uint32_t& a, uint32_t& b) {
  const auto x = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
  a = y[0];
  b = y[1];
}

// Two values rounded to 16 bits each, the first in the lower half.
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const typename T::vec2 v = {(typename T::elem)a, (typename T::elem)b};
  return __builtin_bit_cast(uint32_t, v);
}

// 32 rows of a column, from two tiles' sums, as 16-bit values at p[0..31], those before `end`:
// 16 bytes a lane.
template <class T>
__device__ __forceinline__ void store_rows(typename T::elem* p, int64_t end, bool ok, int lane,
                                           f32x4 v0, f32x4 v1) {
  uint32_t a0 = pack2<T>(v0[0], v0[1]), a1 = pack2<T>(v0[2], v0[3]);
  uint32_t b0 = pack2<T>(v1[0], v1[1]), b1 = pack2<T>(v1[2], v1[3]);
  gather_rows(a0, b0);
  gather_rows(a1, b1);
  if (!ok) return;
  const u32x4v w = {a0, a1, b0, b1};
  const int row = 8 * (lane >> 4);
  if (row + 8 <= end) {
    __builtin_memcpy(p + row, &w, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row + i < end) {
        const uint16_t e = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        __builtin_memcpy(p + row + i, &e, 2);
      }
  }
}

// The stages of a kernel: an array each, so that the compiler knows that loads into one do not touch the
// others and puts no wait before the reads of those; the stages of one operand next to each
// other, so that one address and the reads' constant offsets reach all of them.
#define HOBFLOPS_STAGES2(rows_a, rows_b)                                              \
  __shared__ __align__(1024) uint8_t a0[rows_a * 128], a1[rows_a * 128];              \
  __shared__ __align__(1024) uint8_t b0[rows_b * 128], b1[rows_b * 128];              \
  uint8_t* const sa[2] = {a0, a1};                                                    \
  uint8_t* const sb[2] = {b0, b1}
#define HOBFLOPS_STAGES3(rows_a, rows_b)                                                    \
  __shared__ __align__(1024) uint8_t a0[rows_a * 128], a1[rows_a * 128], a2[rows_a * 128];  \
  __shared__ __align__(1024) uint8_t b0[rows_b * 128], b1[rows_b * 128], b2[rows_b * 128];  \
  uint8_t* const sa[3] = {a0, a1, a2};                                                      \
  uint8_t* const sb[3] = {b0, b1, b2}
#define HOBFLOPS_STAGES4(rows_a, rows_b)                                                        \
  __shared__ __align__(1024) uint8_t a0[rows_a * 128], a1[rows_a * 128], a2[rows_a * 128],      \
      a3[rows_a * 128];                                                                         \
  __shared__ __align__(1024) uint8_t b0[rows_b * 128], b1[rows_b * 128], b2[rows_b * 128],      \
      b3[rows_b * 128];                                                                         \
  uint8_t* const sa[4] = {a0, a1, a2, a3};                                                      \
  uint8_t* const sb[4] = {b0, b1, b2, b3}
#define HOBFLOPS_STAGES6(rows_a, rows_b)                                                        \
  __shared__ __align__(1024) uint8_t a0[rows_a * 128], a1[rows_a * 128], a2[rows_a * 128],      \
      a3[rows_a * 128], a4[rows_a * 128], a5[rows_a * 128];                                     \
  __shared__ __align__(1024) uint8_t b0[rows_b * 128], b1[rows_b * 128], b2[rows_b * 128],      \
      b3[rows_b * 128], b4[rows_b * 128], b5[rows_b * 128];                                     \
  uint8_t* const sa[6] = {a0, a1, a2, a3, a4, a5};                                              \
  uint8_t* const sb[6] = {b0, b1, b2, b3, b4, b5}
#define HOBFLOPS_STAGES8(rows_a, rows_b)                                                        \
  __shared__ __align__(1024) uint8_t a0[rows_a * 128], a1[rows_a * 128], a2[rows_a * 128],      \
      a3[rows_a * 128], a4[rows_a * 128], a5[rows_a * 128], a6[rows_a * 128], a7[rows_a * 128]; \
  __shared__ __align__(1024) uint8_t b0[rows_b * 128], b1[rows_b * 128], b2[rows_b * 128],      \
      b3[rows_b * 128], b4[rows_b * 128], b5[rows_b * 128], b6[rows_b * 128], b7[rows_b * 128]; \
  uint8_t* const sa[8] = {a0, a1, a2, a3, a4, a5, a6, a7};                                      \
  uint8_t* const sb[8] = {b0, b1, b2, b3, b4, b5, b6, b7}

// The gradients' products, D[i][j] with i along a row of the output; kParts weights side by side (the gated
// block's two, a linear layer's one):
//  kWeights 0: dx[t][d], i = d, j = t: A the weights (K-major, w_gate then w_up), B the rows
//    [t][kParts Fp] of dg and du, k = kParts Fp (one part: F rounded up to 8).
//  kWeights 1: dw[f][d], i = d, j = f of kParts Fp: A the rows of x, B those of dg and du, both K-major, k = T.
// Fp is F rounded up to 64 (of one part only F counts); dg and du are zero between F and Fp.
struct GradArgs {
  const void *a[2], *b;
  int64_t lda, ldb, cols, bcols, ni_, nj_, K, F, Fp;  // cols: D rounded up to 8, ni_ = D, nj_: T or kParts Fp; bcols: the width of B's rows, a multiple of 8 (kWeights)
  void* out[2];
  float* part;  // with splits: [splits][nj_][ni_ rounded up to 4]
  int64_t per;  // k of a split, a multiple of 64
  uint32_t ni, nj;
};
template <class T, bool kWeights, int kParts, int BI, int BJ, int WJ, int S>
__device__ __forceinline__ void grad_tile(const GradArgs& p, uint8_t* const (&sa)[S],
                                          uint8_t* const (&sb)[S], uint32_t tile, uint32_t split) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WI = 2, NW = WI * WJ, NI = BI / WI / 16, NJ = BJ / WJ / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t ti, tj;
  tile_of(tile, p.ni, p.nj, ti, tj);
  const int64_t i0 = (int64_t)ti * BI, j0 = (int64_t)tj * BJ;
  const int64_t k0 = (int64_t)split * p.per;
  const int64_t k1 = k0 + p.per < p.K ? k0 + p.per : p.K;
  const int steps = (int)((k1 - k0 + kStepK - 1) / kStepK);
  LoadColumns<BI, NW, kWeights ? 1 : kParts> la;
  std::conditional_t<kWeights, LoadColumns<BJ, NW, 1>, LoadRows<BJ, NW, 1>> lb;
  const void* const bs[1] = {p.b};
  if constexpr (kWeights) {
    const void* const as[1] = {p.a[0]};
    la.start(as, p.lda, p.cols, i0, p.K, p.K, k0, k1, wave, lane);
    lb.start(bs, p.ldb, p.bcols, j0, p.K, p.K, k0, k1, wave, lane);
  } else {
    if constexpr (kParts == 2) {
      la.start(p.a, p.lda, p.cols, i0, p.F, p.Fp, k0, k1, wave, lane);
    } else {
      const void* const as[1] = {p.a[0]};
      la.start(as, p.lda, p.cols, i0, p.F, p.Fp, k0, k1, wave, lane);
    }
    lb.start(bs, p.ldb, p.nj_, j0, k1, k0, wave, lane);
  }
  const auto load = [&](int s) {
    la.load(sa[s], wave);
    lb.load(sb[s], wave);
  };
  const int wi = wave % WI, wj = wave / WI;
  ReadColumns<T, NI, BI> ra;
  std::conditional_t<kWeights, ReadColumns<T, NJ, BJ>, ReadRows<T, NJ, 0>> rb;
  ra.start(wi * NI * 16, lane);
  rb.start(wj * NJ * 16, lane);
  f32x4 acc[NI][NJ] = {};
  if (steps > 0)
    sum_tiles<T, NI, NJ, (BI + BJ) / 8 / NW, S>(acc, sa, sb, ra, rb, load, steps);
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t c = j0 + wj * NJ * 16 + 16 * j + (lane & 15);
    const int64_t half = kWeights && kParts == 2 && c >= p.Fp ? 1 : 0, row = c - half * p.Fp;
    const bool ok = c < p.nj_ && (!kWeights || row < p.F);
#pragma unroll
    for (int i = 0; i < NI; i += 2) {
      const int64_t d = i0 + wi * NI * 16 + 16 * i;
      if (p.part) {
        const int64_t ldp = (p.ni_ + 3) & ~(int64_t)3, at = d + 4 * (lane >> 4);
        float* to = p.part + ((int64_t)split * p.nj_ + c) * ldp + at;
        if (ok && at < p.ni_) *(f32x4*)to = acc[i][j];
        if (ok && at + 16 < p.ni_) *(f32x4*)(to + 16) = acc[i + 1][j];
      } else {
        store_rows<T>((typename T::elem*)p.out[half] + (ok ? row : 0) * p.ni_ + d, p.ni_ - d, ok,
                      lane, acc[i][j], acc[i + 1][j]);
      }
    }
  }
#endif
}

// Sums the splits of a product in their order: bound by reading them, 3.4 to 7 us for up to 32 parts of 77 x 512 and
// 1 x 2048, 37 us for three of 3000 x 4096. (Atomic sums would save it, in an order of their own each time.)
template <class T>
__global__ __launch_bounds__(256) void join_kernel(const float* part, int splits, int64_t rows,
                                                   int64_t cols, typename T::elem* out) {
  const int64_t ldp = (cols + 3) & ~(int64_t)3, n = rows * ldp;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n;
       i += (int64_t)gridDim.x * 1024) {
    f32x4 v = *(const f32x4*)(part + i);
    for (int s = 1; s < splits; ++s) v += *(const f32x4*)(part + s * n + i);
    const int64_t row = i / ldp, col = i - row * ldp;
    const float e[4] = {v[0], v[1], v[2], v[3]};
    store4<T>(out + row * cols, col, cols, e);
  }
}

inline int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
inline unsigned grid_of(int64_t threads, int64_t most) {
  const int64_t n = (threads + 255) / 256;
  return (unsigned)(n < most ? n : most);
}

inline int64_t take(int64_t* total, int64_t bytes) {
  const int64_t at = *total;
  *total += round_up(bytes, 256);
  return at;
}

// Adds a tensor to those that a launch aligns.
inline void add_rows(AlignArgs& a, int i, const void* src, int64_t ld, int64_t rows, void* dst) {
  a.src[i] = src;
  a.dst[i] = dst;
  a.ld[i] = ld;
  for (int j = i; j < 3; ++j) a.rows[j] += rows;
}
template <class T>
void align_rows(const AlignArgs& a, hipStream_t s) {
  if (a.rows[2] > 0) align_kernel<T><<<grid_of(a.rows[2] * a.ldd / 8, 65536), 256, 0, s>>>(a);
}

}  // namespace hobflops
