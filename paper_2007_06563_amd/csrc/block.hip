// Pack and unpack of blocks: narrow floating-point codes with one scale a group
// of a row (activation checkpoints in 8 bits, weights in 4). HBM-bound: a pack
// reads the values once and writes a byte (half a byte) a value, an unpack the
// reverse; the largest magnitude of a group is found in registers, so values
// are not read twice.
//
// A thread holds 8 consecutive values (one 16-byte load of a 16-bit type, two
// of float32) and writes their codes with one store; the 4, 8 or 16 threads of
// a group exchange their largest magnitude. Threads past the row's end, up to
// the end of its last group, hold zeros. A thread's 16 bytes make whole lines a wave
// and leave enough waves to keep HBM busy without a loop.
//
// Measured: 16384 x 4096 bfloat16 in 8 bits: pack 42 us, unpack 33 us, 4.9 and 6.1 TB/s of
// what they read and write (a large copy: 5.1); 4097 x 2731 float32, rows 5 values
// apart and no row aligned: 11 us and 15 us; one row of 4096: 2.5 us, a launch. In 4 bits, groups of 32:
// pack 70 to 75 us (33 at a copy's rate), bound by a division a value, unpack 35 to 16 bits, 46 under
// float32 scales (round_wide_product), 83 to 94 to float32 (60 at a copy's rate).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

constexpr int kPer = 8;        // values a thread
constexpr int kThreads = 256;  // a workgroup

struct BlockParams {
  const void* values;
  uint8_t* codes;
  void* scales;
  int64_t rows, cols, ld, row_bytes;  // row_bytes: codes of a row
  int64_t chunks;                     // threads a row: whole groups
  int group_log, scale;
  bool past;  // unpacked values go past the caches
};

template <class T>
__device__ __forceinline__ void load8(const BlockParams& p, int64_t row, int64_t col, float (&v)[8]) {
  const typename T::elem* src = (const typename T::elem*)p.values + row * p.ld + col;
  if (col + kPer <= p.cols) {  // 16 bytes at a time whatever the alignment
    typename T::elem e[8];
    __builtin_memcpy(e, src, sizeof e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)e[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < p.cols ? (float)src[i] : 0.0f;
  }
}

// The largest of the magnitudes' bits over the 2^(group_log - 3) threads of a group.
__device__ __forceinline__ uint32_t group_max(uint32_t a, int group_log) {
  for (int m = 1; m < 1 << (group_log - 3); m <<= 1) {
    const uint32_t b = (uint32_t)__shfl_xor((int)a, m);
    a = a > b ? a : b;
  }
  return a;
}

template <class T, int kFmt>
__global__ __launch_bounds__(kThreads) void block_pack_kernel(BlockParams p) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = i / p.chunks;
  if (row >= p.rows) return;  // chunks is a multiple of 4: whole groups leave together
  const int64_t col = (i - row * p.chunks) * kPer;
  float v[8];
  load8<T>(p, row, col, v);
  uint32_t a = 0, odd = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = finite_abs(v[j]);
    a = a > b ? a : b;
    odd |= __builtin_isfinite(v[j]) ? 0u : 1u;
  }
  a = group_max(a, p.group_log);
  const int64_t g = col >> p.group_log;
  const int64_t groups = (p.cols + (1 << p.group_log) - 1) >> p.group_log;
  const bool leader = (col & ((1 << p.group_log) - 1)) == 0;
  if (kFmt == kE2M1) {
    // (2, 1) has no code for what is not finite: the group's scale becomes NaN
    odd = group_max(odd, p.group_log);
    float s;
    if (p.scale == HOBFLOPS_SCALE_POW2) {
      const int k = block_scale<kFmt>(a);
      s = pow2f(k);
      if (leader) ((uint8_t*)p.scales)[row * groups + g] = odd ? 255 : (uint8_t)(k + 127);
    } else {
      s = __uint_as_float(a) / 6.0f;
      if (odd) s = __uint_as_float(0x7FC00000u);
      if (p.scale == HOBFLOPS_SCALE_BF16) {
        const __bf16 b = (__bf16)s;
        s = (float)b;
        if (leader) ((__bf16*)p.scales)[row * groups + g] = b;
      } else if (leader) {
        ((float*)p.scales)[row * groups + g] = s;
      }
    }
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, the even code of two; 6 beyond it
      const float n = s > 0.0f ? __builtin_fabsf(v[j]) / s : 0.0f;
      uint32_t c = (n > 0.25f) + (n >= 0.75f) + (n > 1.25f) + (n >= 1.75f) + (n > 2.5f) +
                   (n >= 3.5f) + (n > 5.0f);
      c |= (__float_as_uint(v[j]) >> 31) << 3;
      w |= c << (4 * j);
    }
    uint8_t* dst = p.codes + row * p.row_bytes + col / 2;
    if (col + kPer <= p.cols) {
      __builtin_memcpy(dst, &w, 4);
    } else {
      for (int j = 0; j < 4 && col + 2 * j < p.cols; ++j) dst[j] = (uint8_t)(w >> (8 * j));
    }
  } else {
    const int k = block_scale<kFmt>(a);
    if (leader) ((uint8_t*)p.scales)[row * groups + g] = (uint8_t)(k + 127);
    const float inv = pow2f(-k);
    uint32_t w[2];
    w[0] = encode4<kFmt>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    w[1] = encode4<kFmt>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    uint8_t* dst = p.codes + row * p.row_bytes + col;
    if (col + kPer <= p.cols) {
      __builtin_memcpy(dst, w, 8);
    } else {
      for (int j = 0; j < 8 && col + j < p.cols; ++j) dst[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
  }
}

// A (2, 1) code's value times a float32 scale, rounded to a 16-bit type once: the product needs 25 bits, and
// rounded to float32 first it could fall on the midpoint of two of the type's values. So where it is not
// exact, its float32 takes an odd last place, of the two around it, which keeps it off the midpoints. What
// the float32 is off comes from a multiply-add, or (kSmall) where that could be below 2^-149 from 64 bits.
template <class T, bool kSmall>
__device__ __forceinline__ typename T::elem round_wide_product(float v, float s) {
  const float f = v * s;
  // the sign of product - f (an f that overflowed goes down to the largest float32, which rounds to
  // infinity again)
  float off;
  if constexpr (kSmall) {
    const double d = (double)v * (double)s - (double)f;
    off = d > 0.0 ? 1.0f : d < 0.0 ? -1.0f : 0.0f;
  } else {
    off = __builtin_fmaf(v, s, -f);
  }
  // one step up or down in magnitude from an even last place
  const uint32_t b = __float_as_uint(f), step = (__float_as_uint(off) ^ b) >> 31 ? 0xFFFFFFFFu : 1u;
  const bool move = __builtin_fabsf(off) > 0.0f && !(b & 1u);
  return (typename T::elem)__uint_as_float(move ? b + step : b);
}

template <class T, int kFmt>
__global__ __launch_bounds__(kThreads) void block_unpack_kernel(BlockParams p) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = i / p.chunks;
  if (row >= p.rows) return;
  const int64_t col = (i - row * p.chunks) * kPer;
  if (col >= p.cols) return;
  const int64_t groups = (p.cols + (1 << p.group_log) - 1) >> p.group_log;
  const float s = load_scale(p.scales, row * groups + (col >> p.group_log), p.scale);
  const bool whole = col + kPer <= p.cols;
  float v[8];
  if (kFmt == kE2M1) {
    const uint8_t* src = p.codes + row * p.row_bytes + col / 2;
    uint32_t w = 0;
    if (whole) {
      __builtin_memcpy(&w, src, 4);
    } else {
      for (int j = 0; j < 4 && col + 2 * j < p.cols; ++j) w |= (uint32_t)src[j] << (8 * j);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = decode_e2m1(w >> (4 * j));
  } else {
    const uint8_t* src = p.codes + row * p.row_bytes + col;
    uint32_t w[2] = {0, 0};
    if (whole) {
      __builtin_memcpy(w, src, 8);
    } else {
      for (int j = 0; j < 8 && col + j < p.cols; ++j) w[j >> 2] |= (uint32_t)src[j] << (8 * (j & 3));
    }
    const f32x4 lo = decode4<kFmt>(w[0]), hi = decode4<kFmt>(w[1]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = lo[j];
      v[4 + j] = hi[j];
    }
  }
  typename T::elem* dst = (typename T::elem*)p.values + row * p.ld + col;
  const auto store = [&](auto round) {
    if (whole) {
      typename T::elem e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = round(v[j]);
      // (16384 x 4096 past the caches: 33 us instead of 50; of float32 a lane's 32 bytes are two stores of half lines, which
      // took 4 to 7 % longer in that way)
      if constexpr (sizeof e == 16) {
        u32x4v w;
        __builtin_memcpy(&w, e, 16);
        store16(dst, w, p.past);
      } else {
        __builtin_memcpy(dst, e, sizeof e);
      }
    } else {
      for (int j = 0; j < 8 && col + j < p.cols; ++j) dst[j] = round(v[j]);
    }
  };
  // (the other scales' products with (2, 1) are exact in float32)
  if (kFmt == kE2M1 && sizeof(typename T::elem) == 2 && p.scale == HOBFLOPS_SCALE_F32) {
    if (__all(__builtin_fabsf(s) >= 0x1p-100f))
      store([&](float a) { return round_wide_product<T, false>(a, s); });
    else
      store([&](float a) { return round_wide_product<T, true>(a, s); });
  } else {
    store([&](float a) { return round_product<T>(a, s); });
  }
}

template <class T, int kFmt>
void launch(const BlockParams& p, bool pack, hipStream_t stream) {
  // rows in parts, so that a launch has fewer than 2^31 workgroups of threads
  const int64_t part = ((int64_t)1 << 31) / p.chunks > 0 ? ((int64_t)1 << 31) / p.chunks : 1;
  for (int64_t r = 0; r < p.rows; r += part) {
    BlockParams q = p;
    q.rows = p.rows - r < part ? p.rows - r : part;
    const int64_t groups = (p.cols + (1 << p.group_log) - 1) >> p.group_log;
    const int sbytes = p.scale == HOBFLOPS_SCALE_POW2 ? 1 : p.scale == HOBFLOPS_SCALE_BF16 ? 2 : 4;
    q.values = (const typename T::elem*)p.values + r * p.ld;
    q.codes = p.codes + r * p.row_bytes;
    q.scales = (uint8_t*)p.scales + r * groups * sbytes;
    const unsigned grid = (unsigned)((q.rows * q.chunks + kThreads - 1) / kThreads);
    if (pack)
      block_pack_kernel<T, kFmt><<<grid, kThreads, 0, stream>>>(q);
    else
      block_unpack_kernel<T, kFmt><<<grid, kThreads, 0, stream>>>(q);
  }
}

template <class T>
void launch_fmt(const BlockParams& p, int fmt, bool pack, hipStream_t stream) {
  if (fmt == kE4M3) launch<T, kE4M3>(p, pack, stream);
  if (fmt == kE5M2) launch<T, kE5M2>(p, pack, stream);
  if (fmt == kE2M1) launch<T, kE2M1>(p, pack, stream);
}

hipError_t run(const BlockTensor& t, int fmt, bool pack, hipStream_t stream) {
  BlockParams p{};
  p.values = t.values;
  p.codes = t.codes;
  p.scales = t.scales;
  p.rows = t.rows;
  p.cols = t.cols;
  p.ld = t.ld;
  p.row_bytes = fmt == kE2M1 ? (t.cols + 1) / 2 : t.cols;
  p.group_log = t.group == 32 ? 5 : t.group == 64 ? 6 : 7;
  p.chunks = (t.cols + t.group - 1) / t.group * (t.group / kPer);
  p.scale = t.scale;
  p.past = past_caches(t.rows * t.cols * 2);
  if (t.type == HOBFLOPS_TYPE_F32) launch_fmt<TypeF32>(p, fmt, pack, stream);
  if (t.type == HOBFLOPS_TYPE_BF16) launch_fmt<TypeBF16>(p, fmt, pack, stream);
  if (t.type == HOBFLOPS_TYPE_F16) launch_fmt<TypeF16>(p, fmt, pack, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_pack(const BlockTensor& t, int fmt, hipStream_t stream) {
  return run(t, fmt, true, stream);
}
hipError_t launch_block_unpack(const BlockTensor& t, int fmt, hipStream_t stream) {
  return run(t, fmt, false, stream);
}

}  // namespace hobflops
