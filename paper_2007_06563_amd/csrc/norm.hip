// Layer norm of the rows of a matrix and its gradients:
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps),
//   a = dy w,  dx = rstd (a - mean(a) - xh mean(a xh)) + add,  xh = (x - mean) rstd,
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
// HBM-bound: x, and dy, are read once and stay in registers, a row in one wave or the waves of a
// workgroup. Sums are float32. The variance is of differences from the mean, whose own mean, what the first
// one's rounding left, is taken off again: rows far from 0 keep their digits. Rows whose squares pass float32's
// range are scaled by a power of two.
//
// The sums over rows: a workgroup takes many rows and keeps its part of dw and db in registers; a second
// launch adds the parts in their order (no atomics: the same inputs give the same bits).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "columns.hpp"
#include "lanes.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

struct NormArgs {
  const void *x, *w, *b, *dy, *add;
  void *y, *dx;
  float *mean, *rstd, *part;  // part: [parts][2][cols rounded up to 8]
  int64_t rows, cols, ldx, ldy, ld_add;  // ldy: of y or of dy
  float eps;
};

// Eight values of a row; beyond its end zeros.
template <class T>
__device__ __forceinline__ void load8(const typename T::elem* row, int64_t col, int64_t cols,
                                      typename T::elem (&e)[8]) {
  if (col + 8 <= cols) {  // 16 bytes at a time whatever the alignment
    __builtin_memcpy(e, row + col, sizeof e);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = col + j < cols ? row[col + j] : (typename T::elem)0.0f;
  }
}
template <class T>
__device__ __forceinline__ void load8f(const void* row, int64_t col, int64_t cols, float (&v)[8]) {
  typename T::elem e[8];
  load8<T>((const typename T::elem*)row, col, cols, e);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)e[j];
}
template <class T>
__device__ __forceinline__ void store8(typename T::elem* row, int64_t col, int64_t cols, const float (&v)[8]) {
  if (col + 8 <= cols) {
    typename T::elem e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = (typename T::elem)v[j];
    __builtin_memcpy(row + col, e, sizeof e);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j < cols) row[col + j] = (typename T::elem)v[j];
  }
}

// Sums (or largest values) of a row over its NW waves, the same in every thread; the waves' shares meet in LDS, in one of
// two places, so that one barrier a sum is enough: who writes a place again has passed the barrier of
// the other one, which stands behind all reads of the first.
template <int NW>
__device__ __forceinline__ float2 row_sums(float2 v, float2* lds, int place) {
  v.x = wave_sum(v.x);
  v.y = wave_sum(v.y);
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
template <int NW>
__device__ __forceinline__ float row_max(float v, float2* lds) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, m));
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

// A row's values x[NV][8] become their differences from the mean (0 beyond the end).
template <int NW, int NV>
__device__ __forceinline__ Stats stats_of(float (&x)[NV][8], const int64_t (&col)[NV], int64_t cols, float eps,
                                          float2* lds) {
  const float n = (float)cols;
  float2 s{0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < NV; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) s.x += x[c][j];
  Stats r;
  r.mean = row_sums<NW>(s, lds, 0).x / n;
  s.x = 0.0f;
#pragma unroll
  for (int c = 0; c < NV; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[c][j] = col[c] + j < cols ? x[c][j] - r.mean : 0.0f;
      s.x += x[c][j];
      s.y += x[c][j] * x[c][j];
    }
  s = row_sums<NW>(s, lds, 1);
  r.off = s.x / n;
  float var = s.y / n - r.off * r.off;
  var = var < 0.0f ? 0.0f : var;
  r.rstd = 1.0f / sqrtf(var + eps);
  // (NaN, or 0 for an infinite variance: for the caller)
  return r;
}

template <class T, class W, int NW, int NV>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void norm_kernel(NormArgs p) {
  typedef typename T::elem E;
  constexpr int kRows = NW == 1 ? 4 : 1;  // of a workgroup at a time
  __shared__ float2 lds[2 * NW];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  int64_t col[NV];
  float w[NV][8], b[NV][8];
#pragma unroll
  for (int c = 0; c < NV; ++c) {
    col[c] = ((int64_t)c * NW * 64 + lane) * 8;
    if (p.w)
      load8f<W>(p.w, col[c], p.cols, w[c]);
    else
      for (int j = 0; j < 8; ++j) w[c][j] = 1.0f;
    if (p.b)
      load8f<W>(p.b, col[c], p.cols, b[c]);
    else
      for (int j = 0; j < 8; ++j) b[c][j] = 0.0f;
  }
  for (int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? threadIdx.x >> 6 : 0); row < p.rows;
       row += (int64_t)gridDim.x * kRows) {
    const E* src = (const E*)p.x + row * p.ldx;
    float x[NV][8];
#pragma unroll
    for (int c = 0; c < NV; ++c) load8f<T>(src, col[c], p.cols, x[c]);
    Stats s = stats_of<NW, NV>(x, col, p.cols, p.eps, lds);
    if (!(s.rstd > 0.0f)) {
      // squares beyond float32: the row scaled by a power of two (what is not finite stays NaN)
      float most = 0.0f;
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        load8f<T>(src, col[c], p.cols, x[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(x[c][j]));
      }
      most = row_max<NW>(most, lds);
      const int e = (int)(__float_as_uint(most) >> 23) - 127;
      const float down = pow2f(-(e < 126 ? e : 126));
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[c][j] *= down;
      s = stats_of<NW, NV>(x, col, p.cols, p.eps * down * down, lds);
      if (p.mean && lane == 0) {
        p.mean[row] = (s.mean + s.off) / down;
        p.rstd[row] = s.rstd * down;
      }
    } else if (p.mean && lane == 0) {
      p.mean[row] = s.mean + s.off;
      p.rstd[row] = s.rstd;
    }
    E* dst = (E*)p.y + row * p.ldy;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[c][j] = (x[c][j] - s.off) * s.rstd * w[c][j] + b[c][j];
      store8<T>(dst, col[c], p.cols, x[c]);
    }
  }
}

template <class T, class W, int NW, int NV>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void norm_grad_kernel(NormArgs p) {
  typedef typename T::elem E;
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ float2 lds[2 * NW];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  int64_t col[NV];
  float w[NV][8], dw[NV][8] = {}, db[NV][8] = {};
#pragma unroll
  for (int c = 0; c < NV; ++c) {
    col[c] = ((int64_t)c * NW * 64 + lane) * 8;
    if (p.w)
      load8f<W>(p.w, col[c], p.cols, w[c]);
    else
      for (int j = 0; j < 8; ++j) w[c][j] = 1.0f;
  }
  const float n = (float)p.cols;
  const int64_t first = (int64_t)blockIdx.x * kRows + (NW == 1 ? threadIdx.x >> 6 : 0);
  const int64_t stride = (int64_t)gridDim.x * kRows;
  E xe[NV][8], ge[NV][8];
  float mean = 0.0f, rstd = 0.0f;
  const auto load = [&](int64_t row) {
    mean = p.mean[row];
    rstd = p.rstd[row];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      load8<T>((const E*)p.x + row * p.ldx, col[c], p.cols, xe[c]);
      load8<T>((const E*)p.dy + row * p.ldy, col[c], p.cols, ge[c]);
    }
  };
  if (first < p.rows) load(first);
  int place = 0;
  for (int64_t row = first; row < p.rows; row += stride) {
    float xh[NV][8], a[NV][8], more[NV][8];
    // half of the difference, which stays within range, and twice rstd
    const float half = 0.5f * mean, twice = 2.0f * rstd, r = rstd;
    float2 s{0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = (float)ge[c][j];  // (0 beyond the end)
        xh[c][j] = __builtin_fmaf(0.5f, (float)xe[c][j], -half) * twice;
        a[c][j] = g * w[c][j];
        dw[c][j] += g * xh[c][j];
        db[c][j] += g;
        s.x += a[c][j];
        s.y += a[c][j] * xh[c][j];
      }
    if (p.add) {
#pragma unroll
      for (int c = 0; c < NV; ++c) load8f<T>((const E*)p.add + row * p.ld_add, col[c], p.cols, more[c]);
    }
    // the next row is on its way while this one's sums meet
    if (row + stride < p.rows) load(row + stride);
    s = row_sums<NW>(s, lds, place);
    place ^= 1;
    s.x /= n;
    s.y /= n;
    E* dst = (E*)p.dx + row * p.cols;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        a[c][j] = r * (a[c][j] - s.x - xh[c][j] * s.y);
        if (p.add) a[c][j] += more[c][j];
      }
      store8<T>(dst, col[c], p.cols, a[c]);
    }
  }
  if (p.part) {
    const int64_t wide = (p.cols + 7) & ~(int64_t)7;
    float* to = p.part + first * 2 * wide;
#pragma unroll
    for (int c = 0; c < NV; ++c)
      if (col[c] < p.cols) {
        __builtin_memcpy(to + col[c], dw[c], 32);
        __builtin_memcpy(to + wide + col[c], db[c], 32);
      }
  }
}

// Rows of more than kMostCols values: a workgroup walks the row, three times over (from L2 after the first).
constexpr int64_t kMostCols = 16384;
constexpr int kWide = 16;  // waves

template <class T, class Each>
__device__ __forceinline__ float2 walk(const typename T::elem* row, int64_t cols, float2* lds, int place, Each each) {
  float2 s{0.0f, 0.0f};
  for (int64_t col = (int64_t)threadIdx.x * 8; col < cols; col += kWide * 64 * 8) {
    float v[8];
    load8f<T>(row, col, cols, v);
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
      float var = s.y / n - off * off;
      var = var < 0.0f ? 0.0f : var;
      rstd = 1.0f / sqrtf(var + p.eps * down * down);
      if (rstd > 0.0f || again) break;
      float most = 0.0f;
      for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
        float v[8];
        load8f<T>(src, col, p.cols, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = __builtin_fmaxf(most, __builtin_fabsf(v[j]));
      }
      most = row_max<kWide>(most, lds);
      const int e = (int)(__float_as_uint(most) >> 23) - 127;
      down = pow2f(-(e < 126 ? e : 126));
    }
    if (p.mean && threadIdx.x == 0) {
      p.mean[row] = (mean + off) / down;
      p.rstd[row] = rstd * down;
    }
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float v[8], w[8], b[8];
      load8f<T>(src, col, p.cols, v);
      if (p.w) load8f<W>(p.w, col, p.cols, w);
      if (p.b) load8f<W>(p.b, col, p.cols, b);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = (v[j] * down - mean - off) * rstd * (p.w ? w[j] : 1.0f) + (p.b ? b[j] : 0.0f);
      store8<T>((E*)p.y + row * p.ldy, col, p.cols, v);
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
    const float half = 0.5f * p.mean[row], r = p.rstd[row], twice = 2.0f * r;
    float2 s{0.0f, 0.0f};
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float x[8], g[8], w[8];
      load8f<T>(src, col, p.cols, x);
      load8f<T>(dy, col, p.cols, g);
      if (p.w) load8f<W>(p.w, col, p.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = p.w ? g[j] * w[j] : g[j];
        s.x += a;
        s.y += a * (__builtin_fmaf(0.5f, x[j], -half) * twice);
      }
    }
    s = row_sums<kWide>(s, lds, place);
    place ^= 1;
    s.x /= n;
    s.y /= n;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < p.cols; col += kWide * 64 * 8) {
      float x[8], g[8], w[8], more[8];
      load8f<T>(src, col, p.cols, x);
      load8f<T>(dy, col, p.cols, g);
      if (p.w) load8f<W>(p.w, col, p.cols, w);
      if (p.add) load8f<T>((const E*)p.add + row * p.ld_add, col, p.cols, more);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = p.w ? g[j] * w[j] : g[j];
        x[j] = r * (a - s.x - (__builtin_fmaf(0.5f, x[j], -half) * twice) * s.y) + (p.add ? more[j] : 0.0f);
      }
      store8<T>((E*)p.dx + row * p.cols, col, p.cols, x);
    }
  }
}

// The parts of dw and db of wide rows: 2048 columns and every gridDim.y-th row a workgroup.
template <class T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs p) {
  typedef typename T::elem E;
  const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= p.cols) return;
  float dw[8] = {}, db[8] = {};
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    float x[8], g[8];
    load8f<T>((const E*)p.x + row * p.ldx, col, p.cols, x);
    load8f<T>((const E*)p.dy + row * p.ldy, col, p.cols, g);
    const float half = 0.5f * p.mean[row], twice = 2.0f * p.rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw[j] += g[j] * (__builtin_fmaf(0.5f, x[j], -half) * twice);
      db[j] += g[j];
    }
  }
  const int64_t wide = (p.cols + 7) & ~(int64_t)7;
  float* to = p.part + (int64_t)blockIdx.y * 2 * wide;
  __builtin_memcpy(to + col, dw, 32);
  __builtin_memcpy(to + wide + col, db, 32);
}

// Workgroups of a pass, and with them the parts of a sum over rows.
int64_t forward_groups(int64_t rows, int64_t cols) {
  const int64_t groups = cols <= 1024 ? (rows + 3) / 4 : rows;
  return groups < 2048 ? groups : 2048;
}
int64_t grad_groups(int64_t rows, int64_t cols) {
  const int64_t groups = cols <= 1024 ? (rows + 3) / 4 : rows;
  const int64_t most = cols <= 4096 ? 1024 : cols <= 8192 ? 512 : cols <= kMostCols ? 256 : 128;
  return groups < most ? groups : most;
}
int64_t parts_of(int64_t rows, int64_t cols) { return grad_groups(rows, cols) * (cols <= 1024 ? 4 : 1); }

template <class T, class W>
void forward(const NormArgs& p, hipStream_t s) {
  const unsigned grid = (unsigned)forward_groups(p.rows, p.cols);
  if (p.cols <= 512)
    norm_kernel<T, W, 1, 1><<<grid, 256, 0, s>>>(p);
  else if (p.cols <= 1024)
    norm_kernel<T, W, 1, 2><<<grid, 256, 0, s>>>(p);
  else if (p.cols <= 2048)
    norm_kernel<T, W, 4, 1><<<grid, 256, 0, s>>>(p);
  else if (p.cols <= 4096)
    norm_kernel<T, W, 4, 2><<<grid, 256, 0, s>>>(p);
  else if (p.cols <= 8192)
    norm_kernel<T, W, 8, 2><<<grid, 512, 0, s>>>(p);
  else if (p.cols <= kMostCols)
    norm_kernel<T, W, 16, 2><<<grid, 1024, 0, s>>>(p);
  else
    norm_wide_kernel<T, W><<<grid, kWide * 64, 0, s>>>(p);
}

template <class T, class W>
void backward(const NormArgs& p, void* dw, void* db, hipStream_t s) {
  if (p.rows > 0) {
    const unsigned grid = (unsigned)grad_groups(p.rows, p.cols);
    if (p.cols <= 512) {
      norm_grad_kernel<T, W, 1, 1><<<grid, 256, 0, s>>>(p);
    } else if (p.cols <= 1024) {
      norm_grad_kernel<T, W, 1, 2><<<grid, 256, 0, s>>>(p);
    } else if (p.cols <= 2048) {
      norm_grad_kernel<T, W, 4, 1><<<grid, 256, 0, s>>>(p);
    } else if (p.cols <= 4096) {
      norm_grad_kernel<T, W, 4, 2><<<grid, 256, 0, s>>>(p);
    } else if (p.cols <= 8192) {
      norm_grad_kernel<T, W, 8, 2><<<grid, 512, 0, s>>>(p);
    } else if (p.cols <= kMostCols) {
      norm_grad_kernel<T, W, 16, 2><<<grid, 1024, 0, s>>>(p);
    } else {
      const unsigned walkers = (unsigned)(p.rows < 2048 ? p.rows : 2048);
      norm_grad_wide_kernel<T, W><<<walkers, kWide * 64, 0, s>>>(p);
      if (p.part)
        norm_columns_kernel<T><<<dim3((unsigned)((p.cols + 2047) / 2048), grid), 256, 0, s>>>(p);
    }
  }
  if (dw || db) {
    const int64_t wide = (p.cols + 7) & ~(int64_t)7;
    const int64_t parts = parts_of(p.rows, p.cols);
    launch_column_sums<W>(p.part, parts, 2 * wide, dw, db, p.cols, wide, s);
  }
}

}  // namespace

int64_t norm_backward_workspace(int64_t rows, int64_t cols) {
  return parts_of(rows, cols) * 2 * ((cols + 7) & ~(int64_t)7) * 4;
}

template <class T>
static void norm_of(const LayerNorm& c, const NormArgs& p, bool back, hipStream_t s) {
  if (c.wtype == HOBFLOPS_TYPE_F32)
    back ? backward<T, TypeF32>(p, c.dw, c.db, s) : forward<T, TypeF32>(p, s);
  else
    back ? backward<T, T>(p, c.dw, c.db, s) : forward<T, T>(p, s);
}

static hipError_t norm_run(const LayerNorm& c, bool back, hipStream_t s) {
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
  if (c.type == HOBFLOPS_TYPE_F32) norm_of<TypeF32>(c, p, back, s);
  if (c.type == HOBFLOPS_TYPE_BF16) norm_of<TypeBF16>(c, p, back, s);
  if (c.type == HOBFLOPS_TYPE_F16) norm_of<TypeF16>(c, p, back, s);
  return hipGetLastError();
}

hipError_t launch_norm_forward(const LayerNorm& c, hipStream_t s) { return norm_run(c, false, s); }
hipError_t launch_norm_backward(const LayerNorm& c, hipStream_t s) { return norm_run(c, true, s); }

}  // namespace hobflops
