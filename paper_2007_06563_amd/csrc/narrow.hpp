// Device helpers for 16-bit types, narrow codes with a shared scale and the
// gate's activations.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.hpp"

namespace hobflops {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// The element types: the 16-bit ones with their matrix instruction's operand.
struct TypeF32 {
  typedef float elem;
};
struct TypeBF16 {
  typedef __bf16 elem;
  static constexpr float kMax = 0x1.FEp127f, kStep = 0x1p120f;  // the largest value and its step
  typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
  typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 mfma(vec8 a, vec8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
struct TypeF16 {
  typedef _Float16 elem;
  static constexpr float kMax = 65504.0f, kStep = 32.0f;
  typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
  typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 mfma(vec8 a, vec8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

// A product rounded to a type. For float16 the compiler would join product and
// conversion into a multiply-add with +0, which turns a product of -0 into +0.
template <class T>
__device__ __forceinline__ typename T::elem round_product(float a, float b) {
  float v = a * b;
  if constexpr (sizeof(typename T::elem) == 2) asm("" : "+v"(v));
  return (typename T::elem)v;
}

// 16 bytes to any address of a 16-bit type, or past the caches' reuse. Results of so many bytes go past them that the next call
// finds little of them there anyhow: 16384 x 4096 bfloat16 normed and back 152 us instead of 164, while a norm and two products
// after each other on results of 4 to 67 MB took 2 to 20 % longer in that way (2048 x 4096: 150 us, not 132).
typedef u32x4v Words16 __attribute__((aligned(2)));
__device__ __forceinline__ void store16(void* p, const u32x4v& w, bool past) {
  if (past) {
    // (the compiler would make one store, of the plain kind, of both)
    asm volatile("");
    __builtin_nontemporal_store(w, (Words16*)p);
    asm volatile("");
  } else {
    *(Words16*)p = w;
  }
}
inline bool past_caches(int64_t bytes) { return bytes > (int64_t)64 << 20; }

// 16 bytes moved down by `bits` (128 or more: nothing is left of them), zeros from above.
__device__ __forceinline__ u32x4v shifted_down(const u32x4v& w, uint32_t bits) {
  uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
  lo = bits >= 64 ? hi : lo;
  hi = bits >= 64 ? 0 : hi;
  const uint32_t n = bits & 63;
  lo = lo >> n | (hi << 1) << (63 - n);
  hi >>= n;
  lo = bits >= 128 ? 0 : lo;
  hi = bits >= 128 ? 0 : hi;
  return u32x4v{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The scale exponent k of a group whose largest finite magnitude has the
// float32 bits a: the smallest k >= kMinScale for which the largest magnitude
// times 2^-k does not round beyond the format's largest value. In (4, 3) that
// is 1.75 * 2^8, and 1.8125 * 2^8, the midpoint to the step above, still rounds
// to it (to the even code); in (5, 2) and (2, 1) the midpoint rounds up. Above
// kMinScale every value that codes stand for is a normal float32 and bfloat16.
constexpr int kMinScale = -110;
template <int kFmt>
__device__ __forceinline__ int block_scale(uint32_t a) {
  const uint32_t frac = a & 0x7FFFFFu;
  const int top = kFmt == kE4M3 ? 8 : kFmt == kE5M2 ? 15 : 2;
  const bool over = kFmt == kE4M3   ? frac > 0x680000u
                    : kFmt == kE5M2 ? frac >= 0x700000u
                                    : frac >= 0x600000u;
  const int k = (int)(a >> 23) - 127 - top + (over ? 1 : 0);
  return k > kMinScale ? k : kMinScale;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The bits of |v| if it is finite, else 0.
__device__ __forceinline__ uint32_t finite_abs(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7FFFFFFFu;
  return a < 0x7F800000u ? a : 0u;
}

// Four codes of values already scaled by 2^-k, the first in the low byte. The
// conversion rounds to nearest even, subnormal codes included; infinity, which
// (4, 3) does not have, goes to its NaN.
template <int kFmt>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if (kFmt == kE4M3) {
    const float nan = __uint_as_float(0x7FC00000u);
    a = __builtin_isinf(a) ? nan : a;
    b = __builtin_isinf(b) ? nan : b;
    c = __builtin_isinf(c) ? nan : c;
    d = __builtin_isinf(d) ? nan : d;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
  int w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
}

// The values of four codes, not yet scaled.
template <int kFmt>
__device__ __forceinline__ f32x4 decode4(uint32_t w) {
  f32x2 lo, hi;
  if (kFmt == kE4M3) {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
  }
  return f32x4{lo.x, lo.y, hi.x, hi.y};
}

// The value of a (2, 1) code, unscaled.
__device__ __forceinline__ float decode_e2m1(uint32_t c) {
  const uint32_t m = c & 7u;
  const float v = m < 2 ? 0.5f * (float)m : pow2f((int)(m >> 1) - 1) * (m & 1u ? 1.5f : 1.0f);
  return __uint_as_float(__float_as_uint(v) | (c & 8u) << 28);
}

__device__ __forceinline__ float pow2_scale_of(uint32_t b) {
  return __uint_as_float(b == 255u ? 0x7FC00000u : b == 0u ? 0x00400000u : b << 23);
}
// The scale of a group of 4-bit codes as a float32: a byte's power of two (255:
// NaN), a bfloat16 or a float32.
__device__ __forceinline__ float load_scale(const void* s, int64_t i, int kind) {
  if (kind == HOBFLOPS_SCALE_POW2) return pow2_scale_of(((const uint8_t*)s)[i]);
  if (kind == HOBFLOPS_SCALE_BF16) return (float)((const __bf16*)s)[i];
  return ((const float*)s)[i];
}

// The gate's activation and its derivative.
struct Sigmoid {
  float s, c;  // sigmoid(g) and 1 - sigmoid(g) = sigmoid(-g)
};
// exp(a), a <= 0, to a few units in the last place, subnormal results too: 2^n 2^f with n + f = a / ln 2, f in
// [-1/2, 1/2] from 1 / ln 2 in two parts. A NaN counts as -150. (__expf, 2^(a / ln 2) rounded, loses
// digits with a and everything below 2^-126; expf takes five instructions more for a > 0 and NaN.)
__device__ __forceinline__ float exp_down(float a) {
  a = __builtin_fmaxf(a, -150.0f);
  const float n = __builtin_rintf(a * 1.44269502f);
  const float f = __builtin_fmaf(a, 1.92596299e-8f, __builtin_fmaf(a, 1.44269502f, -n));
  return __builtin_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
}
// From e = exp(-|g|), which does not overflow, so that s and c keep their digits where they are small; the
// reciprocal instruction's last place by one Newton step (1 + e is in [1, 2]; a division would cost ten
// instructions). Of a NaN: numbers, which are multiplied by g.
__device__ __forceinline__ Sigmoid sigmoid_of(float g) {
  const float e = exp_down(-__builtin_fabsf(g)), d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
  const float far = e * r;
  return g < 0.0f ? Sigmoid{far, r} : Sigmoid{r, far};
}
// (erfc: 1 + erf would cancel where the result is small, below -2)
__device__ __forceinline__ float normal_cdf(float g) { return 0.5f * erfcf(g * -0.70710678118654752f); }
__device__ __forceinline__ float gate_act(float g, int act) {
  if (act == HOBFLOPS_GATE_SILU) return g * sigmoid_of(g).s;
  if (act == HOBFLOPS_GATE_GELU) return g * normal_cdf(g);
  return g > 0.0f || g != g ? g : 0.0f;
}
__device__ __forceinline__ void gate_act_grad(float g, int act, float& a, float& da) {
  if (act == HOBFLOPS_GATE_SILU) {
    const Sigmoid v = sigmoid_of(g);
    a = g * v.s;
    da = v.s * (1.0f + g * v.c);
  } else if (act == HOBFLOPS_GATE_GELU) {
    const float p = normal_cdf(g);
    a = g * p;
    da = p + g * exp_down(-0.5f * g * g) * 0.39894228040143268f;
  } else {
    a = g > 0.0f || g != g ? g : 0.0f;
    da = g > 0.0f ? 1.0f : g != g ? g : 0.0f;
  }
}

}  // namespace hobflops
