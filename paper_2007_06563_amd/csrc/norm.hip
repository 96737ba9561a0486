// Layer norm of the rows of a matrix and its gradients:
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps),
//   a = dy w,  dx = rstd (a - mean(a) - xh mean(a xh)) + add,  xh = (x - mean) rstd,
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
// HBM-bound: x, and dy, are read once and stay in registers, a row in one wave or the waves of a
// workgroup. Sums are float32. The variance is of differences from the mean, whose own mean, what the first
// one's rounding left, is taken off again: rows far from 0 keep their digits. Rows whose squares leave float32's
// range, above or below, are scaled by a power of two.
//
// The sums over rows: a workgroup takes many rows and keeps its part of dw and db in registers; a second
// launch adds the parts in their order (no atomics: the same inputs give the same bits).
//
// Measured: 16384 x 4096 bfloat16 forward 46 to 51 us (5.3 to 5.9 TB/s of what it must read and write), backward with a
// gradient to add 94 (5.7) and 5.4 for the parts (25 MB of them); 4097 x 2731 float32 in rows that begin anywhere 20.5 (4.4), 24.3
// (5.5) and 4.0; one row of 4096 3.1, of which the work is one load's latency and two sums'. A large copy: 5.2 TB/s.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "block.hpp"
#include "columns.hpp"
#include "lanes.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

struct NormArgs {
  const void *x, *w, *b, *dy, *add;
  void *y, *dx;
  float *mean, *rstd, *part;  // part: [parts][2][cols]
  int64_t rows, cols, ldx, ldy, ld_add;  // ldy: of y or of dy
  float eps;
  float root;  // the power of two below eps's root, or 0
  bool past;  // y or dx goes past the caches
};

// A thread's values at a time: 16 bytes.
template <class T>
constexpr int kVec = 16 / (int)sizeof(typename T::elem);

// V values of a row; beyond its end zeros.
template <class T, int V>
__device__ __forceinline__ void load_raw(const typename T::elem* row, int64_t col, int64_t cols,
                                         typename T::elem (&e)[V]) {
  if (col + V <= cols) {  // 16 bytes at a time whatever the alignment
    __builtin_memcpy(e, row + col, sizeof e);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = col + j < cols ? row[col + j] : (typename T::elem)0.0f;
  }
}
template <class T, int V>
__device__ __forceinline__ void load_values(const void* row, int64_t col, int64_t cols, float (&v)[V]) {
  typename T::elem e[V];
  load_raw<T, V>((const typename T::elem*)row, col, cols, e);
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = (float)e[j];
}
template <class T, int V>
__device__ __forceinline__ void store_values(typename T::elem* row, int64_t col, int64_t cols, const float (&v)[V]) {
  if (col + V <= cols) {
    typename T::elem e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = (typename T::elem)v[j];
    __builtin_memcpy(row + col, e, sizeof e);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (col + j < cols) row[col + j] = (typename T::elem)v[j];
  }
}
// The 16 bytes of a row that a lane has: of those that would pass the row's end the last ones of the row, so that every
// load and store is a whole one. The first `lead` of their values are another lane's as well: both compute and store
// them alike, and this one leaves them out of the row's sums. (A row has at least as many values; of NC times 16 bytes a
// lane only the last half may pass the end, by the choice of NC.)
template <class T>
struct Chunk {
  int at, lead;
  bool there;  // not all of them another lane's
  __device__ __forceinline__ void start(int col, int cols) {
    constexpr int V = kVec<T>;
    at = col + V <= cols ? col : cols - V;
    lead = col - at;
    there = lead < V;
  }
  __device__ __forceinline__ u32x4v load(const void* row) const {
    u32x4v w;
    __builtin_memcpy(&w, (const typename T::elem*)row + at, 16);
    return w;
  }
  __device__ __forceinline__ void store(void* row, const float (&v)[kVec<T>], bool past) const {
    typename T::elem e[kVec<T>];
#pragma unroll
    for (int j = 0; j < kVec<T>; ++j) e[j] = (typename T::elem)v[j];
    u32x4v w;
    __builtin_memcpy(&w, e, 16);
    if (there) store16((typename T::elem*)row + at, w, past);
  }
};
// Values of a chunk as they count for sums.
template <int NC>
__device__ __forceinline__ float counted(float v, int c, int j, int lead) {
  return c < NC / 2 || j >= lead ? v : 0.0f;
}
template <class T>
__device__ __forceinline__ float value_of(const u32x4v& w, int j) {
  if constexpr (kVec<T> == 4) {
    return __uint_as_float(w[j]);
  } else if constexpr (std::is_same_v<T, TypeBF16>) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
  } else {
    const uint16_t h = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    return (float)__builtin_bit_cast(_Float16, h);
  }
}

// A lane's values of a vector of all columns, or without one a constant.
template <class T, class W, int NC>
__device__ __forceinline__ void load_columns(const void* p, const Chunk<T> (&chunk)[NC], float without,
                                             float (&v)[NC][kVec<T>]) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    typename W::elem e[kVec<T>];
    if (p) __builtin_memcpy(e, (const typename W::elem*)p + chunk[c].at, sizeof e);
#pragma unroll
    for (int j = 0; j < kVec<T>; ++j) v[c][j] = p ? (float)e[j] : without;
  }
}

// Sums (or largest values) of a row over its NW waves, the same in every thread; the waves' shares meet in LDS, in one of
// two places, so that one barrier a sum is enough: who writes a place again has passed the barrier of
// the other one, which stands behind all reads of the first.
template <int NW, int L = 64>
__device__ __forceinline__ float2 row_sums(float2 v, float2* lds, int place) {
  v.x = lanes_sum<L>(v.x);
  v.y = lanes_sum<L>(v.y);
  if constexpr (NW > 1) {
    float2* s = lds + place * NW;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      v.x += s[i].x;
      v.y += s[i].y;
    }
  }
  return v;
}
template <int NW, int L = 64>
__device__ __forceinline__ float row_max(float v, float2* lds) {
#pragma unroll
  for (int m = L / 2; m > 0; m >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, m));
  if constexpr (NW > 1) {
    __syncthreads();  // (a rare path: nothing of the sums' places is relied on)
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6].x = v;
    __syncthreads();
    v = lds[0].x;
#pragma unroll
    for (int i = 1; i < NW; ++i) v = __builtin_fmaxf(v, lds[i].x);
    __syncthreads();
  }
  return v;
}

// The statistics of a row whose values are within float32's range with their squares (and finite: else NaN).
struct Stats {
  float mean, off, rstd;  // the mean is mean + off
};
// Whether they were. A variance (with eps) of more than 2^-120 holds squares to 2^-30 of it, each at most 2^-150 off.
__device__ __forceinline__ bool in_range(float rstd) { return rstd > 0.0f && rstd < 0x1p60f; }
// What a row is scaled by otherwise, from its largest magnitude: that becomes 1 or 2, or less where eps, which is
// scaled twice, would pass the range. (The exponent clamped between both limits would hold one of them in a register, which
// 16-bit rows of 32 to 64 KB do not have: 4096 x 16392 122 us instead of 107.)
__device__ __forceinline__ float scale_down(float most, float root) {
  const int e = (int)(__float_as_uint(__builtin_fmaxf(most, root)) >> 23) - 127;
  return pow2f(-(e < 126 ? e : 126));
}

// From the mean of the differences' squares. What is left of equal values far from 0 is rounding, 2^-24 of the
// differences' mean; a variance of no less than 2^-44 of its square keeps that from growing.
__device__ __forceinline__ float variance(float squares, float off) {
  const float var = squares - off * off, least = off * off * 0x1p-44f;
  return var < least ? least : var;
}
// The same of a row that was scaled by `down`: equal values whose eps is 0 there have the rstd that eps gives.
__device__ __forceinline__ bool equal_values(float rstd, float eps) { return rstd == INFINITY && eps > 0.0f; }

// A row's values become their differences from the mean.
template <class T, int NW, int NC, int L>
__device__ __forceinline__ Stats stats_of(float (&x)[NC][kVec<T>], const Chunk<T> (&chunk)[NC], int64_t cols,
                                          float eps, float2* lds) {
  constexpr int V = kVec<T>;
  const float n = (float)cols;
  float2 s{0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int j = 0; j < V; ++j) s.x += counted<NC>(x[c][j], c, j, chunk[c].lead);
  Stats r;
  r.mean = row_sums<NW, L>(s, lds, 0).x / n;
  s.x = 0.0f;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      x[c][j] -= r.mean;
      const float d = counted<NC>(x[c][j], c, j, chunk[c].lead);
      s.x += d;
      s.y += d * d;
    }
  s = row_sums<NW, L>(s, lds, 1);
  r.off = s.x / n;
  const float var = variance(s.y / n, r.off);
  r.rstd = 1.0f / sqrtf(var + eps);
  // (NaN, 0 for an infinite variance, large for a lost one: for the caller)
  return r;
}

// xh from the saved statistics: the difference passes float32's range where rstd is small enough, its half does not, nor
// twice rstd; where rstd is over 1 neither is halved or doubled, as twice the largest ones would pass it. kRow: the whole wave's
// row is one, and the half takes no vector register.
template <bool kRow>
struct Normed {
  float part, mean, rstd;  // 1/2 or 1; that of the mean; rstd over it
  __device__ __forceinline__ Normed(float m, float r)
      : part(r > 1.0f ? 1.0f : 0.5f), mean(part * m), rstd(r > 1.0f ? r : 2.0f * r) {
    if constexpr (kRow) part = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(part)));
  }
  __device__ __forceinline__ float of(float x) const { return __builtin_fmaf(part, x, -mean) * rstd; }
};

// L lanes of a wave (64 of them but for rows of less than 1 KB), or the NW waves of a workgroup, have a row, a lane NC times 16 bytes of it; the next row is under way
// while a row's sums meet. 32 values a lane leave no registers for w and b, which come from L2 for each
// row (4096 x 16392 bfloat16: 110 us, walked 155).
template <class T, class W, int NW, int NC, int L>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void norm_kernel(NormArgs p) {
  typedef typename T::elem E;
  static_assert(NW == 1 || L == 64);
  constexpr int kRows = NW == 1 ? 256 / L : 1, V = kVec<T>;  // kRows: of a workgroup at a time
  __shared__ float2 lds[2 * NW];
  const int lane = NW == 1 ? threadIdx.x & (L - 1) : threadIdx.x;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? threadIdx.x / L : 0);
  if (row >= p.rows) return;
  Chunk<T> chunk[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) chunk[c].start((c * NW * L + lane) * V, (int)p.cols);
  u32x4v next[NC];
  const auto load = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < NC; ++c) next[c] = chunk[c].load((const E*)p.x + row * p.ldx);
  };
  load(row);
  constexpr bool kHeld = NC * V < 32;  // w and b
  float w[kHeld ? NC : 1][V], b[kHeld ? NC : 1][V];
  if constexpr (kHeld) {
    load_columns<T, W>(p.w, chunk, 1.0f, w);
    load_columns<T, W>(p.b, chunk, 0.0f, b);
  }
  for (; row < p.rows; row += stride) {
    float x[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) x[c][j] = value_of<T>(next[c], j);
    load(row + stride < p.rows ? row + stride : row);  // (of the last row again, rather than a branch)
    Stats s = stats_of<T, NW, NC, L>(x, chunk, p.cols, p.eps, lds);
    if (!in_range(s.rstd)) {
      // the row scaled by a power of two (what is not finite stays NaN)
      float most = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4v v = chunk[c].load((const E*)p.x + row * p.ldx);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          x[c][j] = value_of<T>(v, j);
          most = __builtin_fmaxf(most, __builtin_fabsf(x[c][j]));
        }
      }
      most = row_max<NW, L>(most, lds);
      const float down = scale_down(most, p.root);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) x[c][j] *= down;
      s = stats_of<T, NW, NC, L>(x, chunk, p.cols, p.eps * down * down, lds);
      const bool equal = equal_values(s.rstd, p.eps);
      if (equal) s.rstd = 0.0f;
      if (p.mean && lane == 0) {
        p.mean[row] = (s.mean + s.off) / down;
        p.rstd[row] = equal ? 1.0f / sqrtf(p.eps) : s.rstd * down;
      }
    } else if (p.mean && lane == 0) {
      p.mean[row] = s.mean + s.off;
      p.rstd[row] = s.rstd;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      constexpr int kStep = kHeld ? 1 : 0;
      if constexpr (!kHeld) {
        const Chunk<T> one[1] = {chunk[c]};
        load_columns<T, W>(p.w, one, 1.0f, w);
        load_columns<T, W>(p.b, one, 0.0f, b);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) x[c][j] = (x[c][j] - s.off) * s.rstd * w[c * kStep][j] + b[c * kStep][j];
      chunk[c].store((E*)p.y + row * p.ldy, x[c], p.past);
    }
  }
}

// As norm_kernel; a lane also keeps its columns' parts of dw and db, but where it has 32 values (norm_columns_kernel reads x and
// dy again there: 4096 x 16392 bfloat16: 161 us, walked 303). Sixteen waves with four times 16 bytes a lane have
// registers for neither the next row nor the weights, which come from L2 for each row (2048 x 16384 float32: 137 us, 2.9 TB/s).
template <class T, class W, int NW, int NC, int L>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void norm_grad_kernel(NormArgs p) {
  typedef typename T::elem E;
  static_assert(NW == 1 || L == 64);
  constexpr int kRows = NW == 1 ? 256 / L : 1, V = kVec<T>;
  constexpr bool kAhead = NW * NC < 64, kSums = NC * V < 32;
  __shared__ float2 lds[2 * NW];
  const int lane = NW == 1 ? threadIdx.x & (L - 1) : threadIdx.x;
  const int64_t stride = (int64_t)gridDim.x * kRows;
  const int64_t first = (int64_t)blockIdx.x * kRows + (NW == 1 ? threadIdx.x / L : 0);
  Chunk<T> chunk[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) chunk[c].start((c * NW * L + lane) * V, (int)p.cols);
  const float n = (float)p.cols;
  u32x4v xn[NC], gn[NC], an[NC] = {};  // the next row
  float mean = 0.0f, rstd = 0.0f;
  const auto load = [&](int64_t row) {
    mean = p.mean[row];
    rstd = p.rstd[row];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      xn[c] = chunk[c].load((const E*)p.x + row * p.ldx);
      gn[c] = chunk[c].load((const E*)p.dy + row * p.ldy);
    }
    if (p.add) {
#pragma unroll
      for (int c = 0; c < NC; ++c) an[c] = chunk[c].load((const E*)p.add + row * p.ld_add);
    }
  };
  if (kAhead && first < p.rows) load(first);
  float w[kAhead ? NC : 1][V], dw[kSums ? NC : 1][V] = {}, db[kSums ? NC : 1][V] = {};
  if constexpr (kAhead) load_columns<T, W>(p.w, chunk, 1.0f, w);
  const auto weights = [&](int c) -> const float(&)[V] {
    if constexpr (kAhead) {
      return w[c];
    } else {
      const Chunk<T> one[1] = {chunk[c]};
      load_columns<T, W>(p.w, one, 1.0f, w);
      return w[0];
    }
  };
  int place = 0;
  for (int64_t row = first; row < p.rows; row += stride) {
    if (!kAhead) load(row);
    u32x4v xe[NC], ge[NC], ae[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      xe[c] = xn[c];
      ge[c] = gn[c];
      ae[c] = an[c];
    }
    const Normed<L == 64> normed(mean, rstd);
    const float r = rstd;
    if (kAhead) load(row + stride < p.rows ? row + stride : row);  // (of the last row again, rather than a branch)
    float2 s{0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float(&wc)[V] = weights(c);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = value_of<T>(ge[c], j);
        const float xh = normed.of(value_of<T>(xe[c], j));
        const float a = counted<NC>(g * wc[j], c, j, chunk[c].lead);
        s.x += a;
        s.y += a * counted<NC>(xh, c, j, chunk[c].lead);
      }
    }
    s = row_sums<NW, L>(s, lds, place);
    place ^= 1;
    s.x /= n;
    s.y /= n;
    // (xh and a are formed again: kept through the sums they would take twice the registers)
#pragma unroll
    for (int c = 0; c < NC; ++c) asm("" : "+v"(xe[c]), "+v"(ge[c]), "+v"(ae[c]));
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float(&wc)[V] = weights(c);
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = value_of<T>(ge[c], j);
        const float xh = normed.of(value_of<T>(xe[c], j));
        if constexpr (kSums) {
          dw[c][j] += g * xh;
          db[c][j] += g;
        }
        v[j] = r * (g * wc[j] - s.x - xh * s.y);
        if (p.add) v[j] += value_of<T>(ae[c], j);
      }
      chunk[c].store((E*)p.dx + row * p.cols, v, p.past);
    }
  }
  if (!kSums || !p.part) return;
  if constexpr (NW == 1) {
    // a wave's rows' parts as one, then the four waves', wave after wave
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int m = L; m < 64; m *= 2) {
          dw[c][j] += __shfl_xor(dw[c][j], m);
          db[c][j] += __shfl_xor(db[c][j], m);
        }
    __shared__ float sums[2][NC][V][L];
    for (int i = 1; i < 4; ++i) {
      if ((int)threadIdx.x / L == i * (64 / L)) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            sums[0][c][j][lane] = dw[c][j];
            sums[1][c][j][lane] = db[c][j];
          }
      }
      __syncthreads();
      if (threadIdx.x < L) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            dw[c][j] += sums[0][c][j][lane];
            db[c][j] += sums[1][c][j][lane];
          }
      }
      __syncthreads();
    }
  }
  if constexpr (!kSums) return;
  if (NW > 1 || threadIdx.x < L) {
    float* to = p.part + (int64_t)blockIdx.x * 2 * p.cols;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (chunk[c].there) {
        __builtin_memcpy(to + chunk[c].at, dw[kSums ? c : 0], 4 * V);
        __builtin_memcpy(to + p.cols + chunk[c].at, db[kSums ? c : 0], 4 * V);
      }
  }
}

// Rows of fewer than 16 bytes: a thread has one. (A workgroup for each: a million rows of 4 values 5802 us and 9426 for the gradients, this 9 and 19.)
template <class T>
constexpr int kFew = kVec<T> - 1;  // values at most

template <class T>
__device__ __forceinline__ void load_few(const typename T::elem* p, int n, float (&v)[kFew<T>]) {
#pragma unroll
  for (int j = 0; j < kFew<T>; ++j) v[j] = j < n ? (float)p[j] : 0.0f;
}
template <class T, class W>
__device__ __forceinline__ void load_few_columns(const void* p, int n, float without, float (&v)[kFew<T>]) {
#pragma unroll
  for (int j = 0; j < kFew<T>; ++j) v[j] = p && j < n ? (float)((const typename W::elem*)p)[j] : without;
}

template <class T, class W>
__global__ __launch_bounds__(256) void norm_few_kernel(NormArgs p) {
  typedef typename T::elem E;
  constexpr int M = kFew<T>;
  const int n = (int)p.cols;
  float w[M], b[M];
  load_few_columns<T, W>(p.w, n, 1.0f, w);
  load_few_columns<T, W>(p.b, n, 0.0f, b);
  for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < p.rows; row += (int64_t)gridDim.x * 256) {
    float x[M], down = 1.0f;
    load_few<T>((const E*)p.x + row * p.ldx, n, x);
    Stats r;
    for (int again = 0; again < 2; ++again) {
      float s = 0.0f, off = 0.0f, squares = 0.0f;
#pragma unroll
      for (int j = 0; j < M; ++j) s += x[j];
      r.mean = s / (float)n;
#pragma unroll
      for (int j = 0; j < M; ++j) {
        const float d = j < n ? x[j] - r.mean : 0.0f;
        off += d;
        squares += d * d;
      }
      r.off = off / (float)n;
      r.rstd = 1.0f / sqrtf(variance(squares / (float)n, r.off) + p.eps * down * down);
      if (in_range(r.rstd) || again) break;
      float most = 0.0f;
#pragma unroll
      for (int j = 0; j < M; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(x[j]));
      down = scale_down(most, p.root);
#pragma unroll
      for (int j = 0; j < M; ++j) x[j] *= down;
    }
    const bool equal = down != 1.0f && equal_values(r.rstd, p.eps);
    if (equal) r.rstd = 0.0f;
    if (p.mean) {
      p.mean[row] = (r.mean + r.off) / down;
      p.rstd[row] = equal ? 1.0f / sqrtf(p.eps) : r.rstd * down;
    }
    E* y = (E*)p.y + row * p.ldy;
#pragma unroll
    for (int j = 0; j < M; ++j)
      if (j < n) y[j] = (E)((x[j] - r.mean - r.off) * r.rstd * w[j] + b[j]);
  }
}

template <class T, class W>
__global__ __launch_bounds__(256) void norm_grad_few_kernel(NormArgs p) {
  typedef typename T::elem E;
  constexpr int M = kFew<T>;
  __shared__ float sums[4][2 * M];
  const int n = (int)p.cols;
  float w[M], dw[M] = {}, db[M] = {};
  load_few_columns<T, W>(p.w, n, 1.0f, w);
  for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < p.rows; row += (int64_t)gridDim.x * 256) {
    float x[M], g[M], more[M] = {};
    load_few<T>((const E*)p.x + row * p.ldx, n, x);
    load_few<T>((const E*)p.dy + row * p.ldy, n, g);
    if (p.add) load_few<T>((const E*)p.add + row * p.ld_add, n, more);
    const float r = p.rstd[row];
    const Normed<false> normed(p.mean[row], r);
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int j = 0; j < M; ++j) {
      x[j] = j < n ? normed.of(x[j]) : 0.0f;
      dw[j] += g[j] * x[j];
      db[j] += g[j];
      s0 += g[j] * w[j];
      s1 += g[j] * w[j] * x[j];
    }
    s0 /= (float)n;
    s1 /= (float)n;
    E* dx = (E*)p.dx + row * n;
#pragma unroll
    for (int j = 0; j < M; ++j)
      if (j < n) dx[j] = (E)(r * (g[j] * w[j] - s0 - x[j] * s1) + more[j]);
  }
  if (!p.part) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < M; ++j) {
    dw[j] = wave_sum(dw[j]);
    db[j] = wave_sum(db[j]);
    if (lane == 0) {
      sums[wave][j] = dw[j];
      sums[wave][M + j] = db[j];
    }
  }
  __syncthreads();
  if ((int)threadIdx.x >= 2 * M) return;
  const int j = threadIdx.x < M ? threadIdx.x : threadIdx.x - M;
  if (j < n)
    p.part[((int64_t)blockIdx.x * 2 + (threadIdx.x < M ? 0 : 1)) * n + j] =
        sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x];
}

// Rows of more than 64 KB: a workgroup walks the row, three times over (from L2 after the
// first), at a third of the others' rate.
constexpr int kWide = 16;  // waves

template <class T, class Each>
__device__ __forceinline__ float2 walk(const typename T::elem* row, int64_t cols, float2* lds, int place, Each each) {
  float2 s{0.0f, 0.0f};
  for (int64_t col = (int64_t)threadIdx.x * 8; col < cols; col += kWide * 64 * 8) {
    float v[8];
    load_values<T, 8>(row, col, cols, v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j < cols) each(s, v[j]);
  }
  return row_sums<kWide>(s, lds, place);
}

template <class T, class W>
__global__ __launch_bounds__(kWide * 64) void norm_wide_kernel(NormArgs p) {
  typedef typename T::elem E;
  __shared__ float2 lds[2 * kWide];
  const float n = (float)p.cols;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const E* src = (const E*)p.x + row * p.ldx;
    float down = 1.0f, mean = 0.0f, off = 0.0f, rstd = 0.0f;
    for (int again = 0; again < 2; ++again) {
      mean = walk<T>(src, p.cols, lds, 0, [&](float2& s, float v) { s.x += v * down; }).x / n;
      const float2 s = walk<T>(src, p.cols, lds, 1, [&](float2& s, float v) {
        const float d = v * down - mean;
        s.x += d;
        s.y += d * d;
      });
      off = s.x / n;
      const float var = variance(s.y / n, off);
      rstd = 1.0f / sqrtf(var + p.eps * down * down);
      if (in_range(rstd) || again) break;
      float most = 0.0f;
      for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
        float v[8];
        load_values<T, 8>(src, col, p.cols, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(v[j]));
      }
      most = row_max<kWide>(most, lds);
      down = scale_down(most, p.root);
    }
    const bool equal = down != 1.0f && equal_values(rstd, p.eps);
    if (equal) rstd = 0.0f;
    if (p.mean && threadIdx.x == 0) {
      p.mean[row] = (mean + off) / down;
      p.rstd[row] = equal ? 1.0f / sqrtf(p.eps) : rstd * down;
    }
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float v[8], w[8], b[8];
      load_values<T, 8>(src, col, p.cols, v);
      if (p.w) load_values<W, 8>(p.w, col, p.cols, w);
      if (p.b) load_values<W, 8>(p.b, col, p.cols, b);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = (v[j] * down - mean - off) * rstd * (p.w ? w[j] : 1.0f) + (p.b ? b[j] : 0.0f);
      store_values<T, 8>((E*)p.y + row * p.ldy, col, p.cols, v);
    }
  }
}

template <class T, class W>
__global__ __launch_bounds__(kWide * 64) void norm_grad_wide_kernel(NormArgs p) {
  typedef typename T::elem E;
  __shared__ float2 lds[2 * kWide];
  const float n = (float)p.cols;
  int place = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const E *src = (const E*)p.x + row * p.ldx, *dy = (const E*)p.dy + row * p.ldy;
    const float r = p.rstd[row];
    const Normed<true> normed(p.mean[row], r);
    float2 s{0.0f, 0.0f};
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float x[8], g[8], w[8];
      load_values<T, 8>(src, col, p.cols, x);
      load_values<T, 8>(dy, col, p.cols, g);
      if (p.w) load_values<W, 8>(p.w, col, p.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = p.w ? g[j] * w[j] : g[j];
        s.x += a;
        s.y += a * normed.of(x[j]);
      }
    }
    s = row_sums<kWide>(s, lds, place);
    place ^= 1;
    s.x /= n;
    s.y /= n;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float x[8], g[8], w[8], more[8];
      load_values<T, 8>(src, col, p.cols, x);
      load_values<T, 8>(dy, col, p.cols, g);
      if (p.w) load_values<W, 8>(p.w, col, p.cols, w);
      if (p.add) load_values<T, 8>((const E*)p.add + row * p.ld_add, col, p.cols, more);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = p.w ? g[j] * w[j] : g[j];
        x[j] = r * (a - s.x - normed.of(x[j]) * s.y) + (p.add ? more[j] : 0.0f);
      }
      store_values<T, 8>((E*)p.dx + row * p.cols, col, p.cols, x);
    }
  }
}

// The parts of dw and db of rows that nobody has in registers: 2048 columns and every gridDim.y-th row a workgroup.
template <class T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs p) {
  typedef typename T::elem E;
  const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= p.cols) return;
  float dw[8] = {}, db[8] = {};
  const auto add = [&](const float (&x)[8], const float (&g)[8], int64_t row) {
    const Normed<true> normed(p.mean[row], p.rstd[row]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw[j] += g[j] * normed.of(x[j]);
      db[j] += g[j];
    }
  };
  int64_t row = blockIdx.y;
  if (col + 8 <= p.cols) {
    // four rows under way
    for (; row + 3 * (int64_t)gridDim.y < p.rows; row += 4 * (int64_t)gridDim.y) {
      E x[4][8], g[4][8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = row + i * (int64_t)gridDim.y;
        __builtin_memcpy(x[i], (const E*)p.x + r * p.ldx + col, sizeof x[i]);
        __builtin_memcpy(g[i], (const E*)p.dy + r * p.ldy + col, sizeof g[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8], d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = (float)x[i][j];
          d[j] = (float)g[i][j];
        }
        add(v, d, row + i * (int64_t)gridDim.y);
      }
    }
  }
  for (; row < p.rows; row += gridDim.y) {
    float x[8], g[8];
    load_values<T, 8>((const E*)p.x + row * p.ldx, col, p.cols, x);
    load_values<T, 8>((const E*)p.dy + row * p.ldy, col, p.cols, g);
    add(x, g, row);
  }
  float* to = p.part + (int64_t)blockIdx.y * 2 * p.cols + col;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (col + j < p.cols) {
      to[j] = dw[j];
      to[p.cols + j] = db[j];
    }
}

// The kernels' shapes: a row in up to `chunks` times 16 bytes, two a lane (beyond 32 KB four), the
// more waves the longer it is. (Four a lane, 4097 x 2731 float32: backward 40 us, two waves on a SIMD; two a lane 28.
// Two waves with two each rather than four with one: 2^25 bfloat16 values in rows of 2048 23 us instead of 31, of 1536 28 instead
// of 37. Short rows share a wave: in rows of 64 27 us, with a wave each 166.)
struct Shape {
  int waves;
  int64_t chunks;  // at most
};
constexpr Shape kShapes[] = {{1, 64}, {1, 128}, {2, 256}, {4, 512}, {8, 1024}, {16, 2048}, {16, 4096}};
constexpr int kWalk = 7, kThread = 8;  // none of them: rows are walked, or a thread's
int shape_of(int64_t cols, int type) {
  const int64_t chunks = (cols + (type == HOBFLOPS_TYPE_F32 ? 3 : 7)) / (type == HOBFLOPS_TYPE_F32 ? 4 : 8);
  if (cols < (type == HOBFLOPS_TYPE_F32 ? 4 : 8)) return kThread;  // (no whole 16 bytes)
  int i = 0;
  while (i < kWalk && chunks > kShapes[i].chunks) ++i;
  return i;
}
// Lanes of a row of up to 64 times 16 bytes.
int lanes_of(int64_t cols, int type) {
  const int64_t chunks = (cols + (type == HOBFLOPS_TYPE_F32 ? 3 : 7)) / (type == HOBFLOPS_TYPE_F32 ? 4 : 8);
  int lanes = 4;
  while (lanes < 64 && lanes < chunks) lanes *= 2;
  return lanes;
}
// Waves of a row. Forward, float32 rows of 2 to 32 KB have half as many with four times 16 bytes a lane: the fewer lanes
// without values the better (4097 x 2731: 17.7 us instead of 20, 4095 x 4097: 27 instead of 37).
int waves_of(int shape, int type, bool grad) {
  const int waves = kShapes[shape].waves;
  return type == HOBFLOPS_TYPE_F32 && !grad && shape >= 2 && shape <= 5 ? waves / 2 : waves;
}
// Whether the sums over rows have a launch of their own.
bool columns_apart(int shape, int type) { return shape == kWalk || (shape == 6 && type != HOBFLOPS_TYPE_F32); }
// Backward, eight waves of 16-bit values, which are twice as many a lane, would be one workgroup on a CU, or two whose
// registers spill (8192 x 8192 bfloat16: 226 us); sixteen waves with half of a lane's values take 96.
bool wide_grad(int shape, int type) { return shape == 4 && type != HOBFLOPS_TYPE_F32; }
// Workgroups of a pass: about as many as are on the chip at a time (backward: three waves on a SIMD, four of
// those with 8 or 16 in a workgroup).
int64_t groups_of(int64_t rows, int64_t cols, int type, bool grad) {
  const int i = shape_of(cols, type);
  if (i == kWalk) return rows < 512 ? rows : 512;
  if (i == kThread) return rows < 256 * 1024 ? (rows + 255) / 256 : 1024;
  const int waves = waves_of(i, type, grad);
  const int64_t each = i == 0 ? 256 / lanes_of(cols, type) : waves == 1 ? 4 : 1, groups = (rows + each - 1) / each;
  const int64_t most = !grad       ? (waves == 16 ? 512 : 2048)
                       : waves == 2 ? 1536
                       : waves <= 4 ? 768
                       : waves == 8 && !wide_grad(i, type) ? 512
                                                           : 256;
  return groups < most ? groups : most;
}
// The parts of the sums over rows: one a workgroup.
constexpr int64_t kWideParts = 128;
int64_t parts_of(int64_t rows, int64_t cols, int type) {
  if (columns_apart(shape_of(cols, type), type)) return rows < kWideParts ? rows : kWideParts;
  return groups_of(rows, cols, type, true);
}

template <class T>
constexpr int kType = kVec<T> == 4 ? HOBFLOPS_TYPE_F32 : HOBFLOPS_TYPE_BF16;  // (either 16-bit type)

template <class T, class W, int NW, int NC, int L = 64>
void launch_grad(const NormArgs& p, hipStream_t s) {
  norm_grad_kernel<T, W, NW, NC, L>
      <<<(unsigned)groups_of(p.rows, p.cols, kType<T>, true), NW == 1 ? 256 : NW * 64, 0, s>>>(p);
}
template <class T, class W, int NW, int NC, int L = 64>
void launch_forward(const NormArgs& p, hipStream_t s) {
  norm_kernel<T, W, NW, NC, L>
      <<<(unsigned)groups_of(p.rows, p.cols, kType<T>, false), NW == 1 ? 256 : NW * 64, 0, s>>>(p);
}
template <class T, class W, int NW, int NC, int L = 64>
void launch(const NormArgs& p, bool grad, hipStream_t s) {
  if constexpr (NW != 8 || kVec<T> == 4) {
    if (grad) return launch_grad<T, W, NW, NC, L>(p, s);
  }
  if constexpr (kVec<T> == 4 && NW >= 2 && NC == 2)
    launch_forward<T, W, NW / 2, 4>(p, s);
  else
    launch_forward<T, W, NW, NC, L>(p, s);
}
template <class T, class W>
void launch_rows(const NormArgs& p, bool grad, hipStream_t s) {
  if (p.rows == 0) return;
  switch (shape_of(p.cols, kType<T>)) {
    case 0:
      switch (lanes_of(p.cols, kType<T>)) {
        case 4: return launch<T, W, 1, 1, 4>(p, grad, s);
        case 8: return launch<T, W, 1, 1, 8>(p, grad, s);
        case 16: return launch<T, W, 1, 1, 16>(p, grad, s);
        case 32: return launch<T, W, 1, 1, 32>(p, grad, s);
        default: return launch<T, W, 1, 1>(p, grad, s);
      }
    case 1: return launch<T, W, 1, 2>(p, grad, s);
    case 2: return launch<T, W, 2, 2>(p, grad, s);
    case 3: return launch<T, W, 4, 2>(p, grad, s);
    case 4:
      if constexpr (kVec<T> == 8) {
        if (grad) return launch_grad<T, W, 16, 1>(p, s);
      }
      return launch<T, W, 8, 2>(p, grad, s);
    case 5: return launch<T, W, 16, 2>(p, grad, s);
    case 6:
      launch<T, W, 16, 4>(p, grad, s);
      break;
    case kThread: {
      const unsigned grid = (unsigned)groups_of(p.rows, p.cols, kType<T>, grad);
      if (grad)
        norm_grad_few_kernel<T, W><<<grid, 256, 0, s>>>(p);
      else
        norm_few_kernel<T, W><<<grid, 256, 0, s>>>(p);
      return;
    }
    default: {
      const unsigned grid = (unsigned)groups_of(p.rows, p.cols, kType<T>, grad);
      if (grad)
        norm_grad_wide_kernel<T, W><<<grid, kWide * 64, 0, s>>>(p);
      else
        norm_wide_kernel<T, W><<<grid, kWide * 64, 0, s>>>(p);
    }
  }
  if (grad && p.part && columns_apart(shape_of(p.cols, kType<T>), kType<T>))
    norm_columns_kernel<T><<<dim3((unsigned)((p.cols + 2047) / 2048), (unsigned)parts_of(p.rows, p.cols, kType<T>)), 256, 0,
                             s>>>(p);
}

template <class T, class W>
void run_types(const LayerNorm& c, const NormArgs& p, bool grad, hipStream_t s) {
  launch_rows<T, W>(p, grad, s);
  if (!grad || !(c.dw || c.db)) return;
  launch_column_sums<W>(p.part, parts_of(p.rows, p.cols, kType<T>), 2 * p.cols, c.dw, c.db, p.cols, p.cols, s);
}
template <class T>
void run_type(const LayerNorm& c, const NormArgs& p, bool grad, hipStream_t s) {
  if (c.wtype == HOBFLOPS_TYPE_F32)
    run_types<T, TypeF32>(c, p, grad, s);
  else
    run_types<T, T>(c, p, grad, s);
}

hipError_t run(const LayerNorm& c, bool grad, hipStream_t s) {
  NormArgs p{};
  p.x = c.x;
  p.w = c.w;
  p.b = c.b;
  p.dy = c.dy;
  p.add = c.add;
  p.y = c.y;
  p.dx = c.dx;
  p.mean = c.mean;
  p.rstd = c.rstd;
  p.part = c.dw || c.db ? (float*)c.workspace : nullptr;
  p.rows = c.rows;
  p.cols = c.cols;
  p.ldx = c.ldx;
  p.ldy = c.ldy;
  p.ld_add = c.ld_add;
  p.eps = (float)c.eps;
  p.root = p.eps > 0.0f ? ldexpf(1.0f, ilogbf(p.eps) >> 1) : 0.0f;
  p.past = past_caches(c.rows * c.cols * (c.type == HOBFLOPS_TYPE_F32 ? 4 : 2));
  if (c.type == HOBFLOPS_TYPE_F32) run_type<TypeF32>(c, p, grad, s);
  if (c.type == HOBFLOPS_TYPE_BF16) run_type<TypeBF16>(c, p, grad, s);
  if (c.type == HOBFLOPS_TYPE_F16) run_type<TypeF16>(c, p, grad, s);
  return hipGetLastError();
}

}  // namespace

int64_t norm_backward_workspace(int64_t rows, int64_t cols, int type) {
  return parts_of(rows, cols, type) * 2 * cols * 4;
}
hipError_t launch_norm_forward(const LayerNorm& c, hipStream_t s) { return run(c, false, s); }
hipError_t launch_norm_backward(const LayerNorm& c, hipStream_t s) { return run(c, true, s); }

}  // namespace hobflops
