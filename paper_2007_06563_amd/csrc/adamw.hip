// An AdamW step over many tensors at once, with the moments in float32 or in 8 bits:
//   g' = scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr decay) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// HBM-bound: every tensor is read and written once, in one launch for up to 64 of them (their
// addresses are kernel arguments). A thread takes 4 values at a time: 138 M values with bfloat16 gradients and copies
// 715 us (5.4 TB/s of 28 bytes a value), with 8-bit states 418 (5.3, of 16.1 bytes); 2.16 M with float32 gradients 11.8, from
// the last cache; forty tensors of 0.8 M values 8.1, a launch and one round's latency.
//
// All operations are float32 ones, each rounded (no multiply-add takes two of them together), so
// that the results are those of the formula written with elementary operations, bit for bit.
//
// 8-bit states are blocks of 32 values under a power of two: m in codes of the format, v by its
// square root r, which halves the exponents' range. The scale is the smallest for which the largest
// value of a group is no larger than the format's. Rounding to nearest would hold the states where
// they are: v moves by 1 - b2 (0.1 %) a step, a code of r by 12 to 25 % of r^2. So a value between
// two codes goes to one of them at random: m so that its mean stays m, r so that the mean of r^2
// stays v (the mean of r instead would let v grow by the variance of r, more than 1 - b2 of it
// a step). A root that is not zero keeps the least code at least: m / (0 + eps) would be large.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "block.hpp"
#include "lanes.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;        // values a thread at a time: 16 bytes of float32, whole lines a wave
constexpr int kTensors = 64;   // a launch: 3 KB of arguments

struct Tensor {
  float* p;
  const void* g;
  void* copy;
  int64_t n, at;  // values; the place of the first one in the states
};
struct Args {
  Tensor t[kTensors];
  uint32_t first[kTensors];  // workgroup of each; of those that there are not 2^32 - 1
  void *m, *v;
  uint8_t *m_scales, *v_scales;
  const float *lr_at, *scale_at, *skip_at;  // null: the values below
  const int64_t* step_at;
  double lr, decay, log_b1, log_b2;
  uint64_t seed;
  float b1, c1, b2, c2, eps, keep, rate, root, scale;  // c: 1 - b; keep: 1 - lr decay
  uint32_t key;
  int count, copy_type;
};

// Rounds of a workgroup, kThreads * kPer values each.
template <bool kStream>
constexpr int kRounds = kStream ? 8 : 1;

// 32 bits stirred: two rounds of a fold and an odd factor (digits of the square roots of 3 and 2).
__host__ __device__ __forceinline__ uint32_t stirred(uint32_t x) {
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  x = (x ^ (x >> 13)) * 0x6A09E667u;
  return x ^ (x >> 16);
}
// The start of a step's counter.
__host__ __device__ __forceinline__ uint32_t step_key(int64_t step, uint64_t seed) {
  uint32_t k = stirred((uint32_t)step);
  k = stirred(k ^ (uint32_t)((uint64_t)step >> 32));
  k = stirred(k ^ (uint32_t)seed);
  return stirred(k ^ (uint32_t)(seed >> 32));
}
// The random bits of the value at a place (below 2^32 places; beyond them the key moves on).
__device__ __forceinline__ uint32_t bits_of(uint32_t key, int64_t place) {
  return stirred((uint32_t)place * 0x9E3779B9u + (key ^ (uint32_t)(place >> 32) * 0x6A09E667u));
}

// A thread's values, `left` of them; zeros beyond.
template <class G, bool kStream>
__device__ __forceinline__ void load_values(const typename G::elem* src, int64_t left, float (&v)[kPer]) {
  typedef typename G::elem E;
  if (left >= kPer) {
    typedef uint32_t Words __attribute__((ext_vector_type(kPer * sizeof(E) / 4), aligned(sizeof(E))));
    const Words w = kStream ? __builtin_nontemporal_load((const Words*)src) : *(const Words*)src;
    E e[kPer];
    __builtin_memcpy(e, &w, sizeof e);
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = (float)e[j];
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = j < left ? (float)src[j] : 0.0f;
  }
}
template <class G, bool kStream>
__device__ __forceinline__ void store_values(typename G::elem* dst, int64_t left, const float (&v)[kPer]) {
  typedef typename G::elem E;
  if (left >= kPer) {
    E e[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) e[j] = (E)v[j];
    typedef uint32_t Words __attribute__((ext_vector_type(kPer * sizeof(E) / 4), aligned(sizeof(E))));
    Words w;
    __builtin_memcpy(&w, e, sizeof e);
    if (kStream)
      __builtin_nontemporal_store(w, (Words*)dst);
    else
      *(Words*)dst = w;
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j < left) dst[j] = (E)v[j];
  }
}

template <int kFmt>
__device__ __forceinline__ void decode_values(const uint8_t* codes, uint8_t scale, float (&v)[kPer]) {
  uint32_t w;
  __builtin_memcpy(&w, codes, 4);
  const float s = pow2_scale_of(scale);
  const f32x4 d = decode4<kFmt>(w);
#pragma unroll
  for (int j = 0; j < kPer; ++j) v[j] = d[j] * s;
}

// The smallest scale exponent, at least kMinScale, under which the largest of eight threads' values is no
// larger than the format's largest, 1.75 * 2^8 or 1.75 * 2^15.
template <int kFmt>
__device__ __forceinline__ int group_scale(const float (&v)[kPer]) {
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) a = max(a, finite_abs(v[j]));
  a = max(a, row_xor<1>(a));
  a = max(a, row_xor<2>(a));
  a = max(a, row_xor<3>(a));
  const int k = (int)(a >> 23) - 127 - (kFmt == kE4M3 ? 8 : 15) + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return k > kMinScale ? k : kMinScale;
}

// A scaled magnitude's place among the codes: n / step and step, the distance of the codes there.
template <int kFmt>
__device__ __forceinline__ float in_steps(float n, float& step) {
  constexpr int kLow = kFmt == kE4M3 ? -6 : -14, kFrac = kFmt == kE4M3 ? 3 : 2;
  int e = (int)(__float_as_uint(n) >> 23) - 127;
  e = e > kLow ? e : kLow;
  step = pow2f(e - kFrac);
  return n * pow2f(kFrac - e);
}

template <int kFmt>
__device__ __forceinline__ void store_codes(uint8_t* codes, const float (&q)[kPer]) {
  const uint32_t w = encode4<kFmt>(q[0], q[1], q[2], q[3]);
  __builtin_memcpy(codes, &w, 4);
}

// The factors that depend on the step, where it or the rate stands on the device.
__device__ __forceinline__ void factors_of(const Args& a, float& keep, float& rate, float& root, uint32_t& key) {
  keep = a.keep;
  rate = a.rate;
  root = a.root;
  key = a.key;
  if (!a.lr_at && !a.step_at) return;
  const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
  keep = (float)(1.0 - lr * a.decay);
  // (without step_at log_b1 and log_b2 are those of the powers, and t is 1)
  const int64_t t = a.step_at ? *a.step_at : 1;
  rate = (float)(lr / -expm1((double)t * a.log_b1));
  root = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
  if (a.step_at) key = step_key(t, a.seed);
}

// kStream: so many values that they do not stay in the last cache from step to step: past the caches, and eight rounds a
// workgroup. (2.16 M values, 60 MB, in this way 21 us, otherwise 13; 138 M values 2 % less in this way.)
template <int kFmt, class G, bool kStream>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Args a) {
#pragma clang fp contract(off)
  if (a.skip_at && !(*a.skip_at == 0.0f)) return;
  // the last tensor that begins at or before this workgroup: a lane looks at one
  static_assert(kTensors == 64);
  const int last = __builtin_popcountll(__ballot(a.first[threadIdx.x & 63] <= blockIdx.x)) - 1;
  const uint32_t first = a.first[last];
  const Tensor t = a.t[last];
  float keep, rate, root;
  uint32_t key;
  factors_of(a, keep, rate, root, key);
  const float scale = a.scale_at ? *a.scale_at : a.scale;
  int64_t i = (int64_t)(blockIdx.x - first) * kRounds<kStream> * (kThreads * kPer) + threadIdx.x * kPer;
  for (int round = 0; round < kRounds<kStream>; ++round, i += kThreads * kPer) {
    // (eight threads of a group of 32 leave together)
    if (i >= ((t.n + 31) & ~(int64_t)31)) return;
    const int64_t left = t.n - i, at = t.at + i;
    float p[kPer], g[kPer], m[kPer], v[kPer];
    load_values<TypeF32, kStream>(t.p + i, left, p);
    load_values<G, kStream>((const typename G::elem*)t.g + i, left, g);
    if constexpr (kFmt < 0) {
      load_values<TypeF32, kStream>((const float*)a.m + at, left, m);
      load_values<TypeF32, kStream>((const float*)a.v + at, left, v);
    } else {
      decode_values<kFmt>((const uint8_t*)a.m + at, a.m_scales[at >> 5], m);
      decode_values<kFmt>((const uint8_t*)a.v + at, a.v_scales[at >> 5], v);
#pragma unroll
      for (int j = 0; j < kPer; ++j) v[j] = v[j] * v[j];
    }
    float r[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float d = g[j] * scale;
      m[j] = m[j] * a.b1 + d * a.c1;
      v[j] = v[j] * a.b2 + d * d * a.c2;
      r[j] = sqrtf(v[j]);
      p[j] = p[j] * keep - m[j] / (r[j] * root + a.eps) * rate;
    }
    store_values<TypeF32, kStream>(t.p + i, left, p);
    if (t.copy) {
      if (a.copy_type == HOBFLOPS_TYPE_BF16)
        store_values<TypeBF16, kStream>((__bf16*)t.copy + i, left, p);
      else
        store_values<TypeF16, kStream>((_Float16*)t.copy + i, left, p);
    }
    if constexpr (kFmt < 0) {
      store_values<TypeF32, kStream>((float*)a.m + at, left, m);
      store_values<TypeF32, kStream>((float*)a.v + at, left, v);
    } else {
      if (left < kPer) {  // behind the tensor's end, up to its last group's: zeros
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (j >= left) m[j] = r[j] = v[j] = 0.0f;
      }
      const int km = group_scale<kFmt>(m), kr = group_scale<kFmt>(r);
      if ((at & 31) == 0) {
        a.m_scales[at >> 5] = (uint8_t)(km + 127);
        a.v_scales[at >> 5] = (uint8_t)(kr + 127);
      }
      const float sm = pow2f(-km), sr = pow2f(-kr);
      constexpr float kLeast = kFmt == kE4M3 ? 0x1p-9f : 0x1p-16f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t bits = bits_of(key, at + j);
        float step;
        const float n = in_steps<kFmt>(__builtin_fabsf(m[j]) * sm, step), whole = floorf(n);
        const float um = ((float)(bits & 0xFFFFu) + 0.5f) * 0x1p-16f;
        m[j] = __builtin_copysignf((n - whole > um ? whole + 1.0f : whole) * step, m[j]);
        const float ur = ((float)(bits >> 16) + 0.5f) * 0x1p-16f;
        const float y = r[j] * sr;
        const float below = floorf(in_steps<kFmt>(y, step)) * step, above = below + step;
        const float b2 = below * below;
        float q = v[j] * sr * sr - b2 > ur * (above * above - b2) ? above : below;
        if (y > 0.0f && q < kLeast) q = kLeast;
        r[j] = __builtin_isfinite(y) ? q : __builtin_fabsf(y);  // (a NaN may have a sign)
      }
      store_codes<kFmt>((uint8_t*)a.m + at, m);
      store_codes<kFmt>((uint8_t*)a.v + at, r);
    }
  }
}

template <int kFmt, class G>
void launch(const Args& a, bool stream, uint32_t grid, hipStream_t s) {
  if (stream)
    adamw_kernel<kFmt, G, true><<<grid, kThreads, 0, s>>>(a);
  else
    adamw_kernel<kFmt, G, false><<<grid, kThreads, 0, s>>>(a);
}
template <int kFmt>
void launch_type(const Args& a, int type, bool stream, uint32_t grid, hipStream_t s) {
  if (type == HOBFLOPS_TYPE_F32) launch<kFmt, TypeF32>(a, stream, grid, s);
  if (type == HOBFLOPS_TYPE_BF16) launch<kFmt, TypeBF16>(a, stream, grid, s);
  if (type == HOBFLOPS_TYPE_F16) launch<kFmt, TypeF16>(a, stream, grid, s);
}

}  // namespace

hipError_t launch_adamw(const hobflops_adamw_desc& d, const hobflops_adamw_tensor* tensors, int count,
                        int fmt, const AdamwState& state, hipStream_t stream) {
  Args a{};
  a.m = state.m;
  a.v = state.v;
  a.m_scales = state.m_scales;
  a.v_scales = state.v_scales;
  a.lr_at = d.lr_at;
  a.step_at = d.step_at;
  a.scale_at = d.grad_scale_at;
  a.skip_at = d.skip_at;
  a.lr = d.lr;
  a.decay = d.weight_decay;
  const double t = d.step_at ? 1.0 : (double)d.step;
  a.log_b1 = log(d.beta1) * t;  // (of 0: minus infinity, whose power is 0)
  a.log_b2 = log(d.beta2) * t;
  a.seed = d.seed;
  a.b1 = (float)d.beta1;
  a.c1 = (float)(1.0 - d.beta1);
  a.b2 = (float)d.beta2;
  a.c2 = (float)(1.0 - d.beta2);
  a.eps = (float)d.eps;
  a.keep = (float)(1.0 - d.lr * d.weight_decay);
  a.rate = (float)(d.lr / -expm1(a.log_b1));
  a.root = (float)(1.0 / sqrt(-expm1(a.log_b2)));
  a.scale = (float)d.grad_scale;
  a.key = step_key(d.step, d.seed);
  a.copy_type = d.copy_type;
  int64_t all = 0;
  for (int i = 0; i < count; ++i) all += tensors[i].g ? tensors[i].n : 0;
  const bool large = all > (int64_t)1 << 22;  // 117 MB in float32, of which the last cache holds 256
  const int64_t chunk = (large ? kRounds<true> : kRounds<false>) * kThreads * kPer;
  int64_t at = 0;
  uint64_t grid = 0;
  const auto flush = [&] {
    if (a.count == 0) return;
    if (fmt == kE4M3)
      launch_type<kE4M3>(a, d.grad_type, large, (uint32_t)grid, stream);
    else if (fmt == kE5M2)
      launch_type<kE5M2>(a, d.grad_type, large, (uint32_t)grid, stream);
    else
      launch_type<-1>(a, d.grad_type, large, (uint32_t)grid, stream);
    a.count = 0;
    grid = 0;
    for (int i = 0; i < kTensors; ++i) a.first[i] = UINT32_MAX;
  };
  for (int i = 0; i < kTensors; ++i) a.first[i] = UINT32_MAX;
  for (int i = 0; i < count; ++i) {
    const hobflops_adamw_tensor& c = tensors[i];
    // a part of a tensor a launch, so that a launch has fewer than 2^32 threads
    const int64_t part = (int64_t)1 << 34;
    for (int64_t o = 0; c.g && o < c.n; o += part) {
      const int64_t n = c.n - o < part ? c.n - o : part;
      const uint64_t groups = (uint64_t)((n + chunk - 1) / chunk);
      if (a.count == kTensors || grid + groups >= (uint64_t)1 << 24) flush();
      a.first[a.count] = (uint32_t)grid;
      Tensor& e = a.t[a.count++];
      const int gb = d.grad_type == HOBFLOPS_TYPE_F32 ? 4 : 2;
      e.p = c.p + o;
      e.g = (const uint8_t*)c.g + o * gb;
      e.copy = c.copy ? (uint8_t*)c.copy + o * 2 : nullptr;
      e.n = n;
      e.at = at + o;
      grid += groups;
    }
    at += (c.n + 31) & ~(int64_t)31;
  }
  flush();
  return hipGetLastError();
}

}  // namespace hobflops
