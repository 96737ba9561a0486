// Products of a few tokens with 4-bit weights under group scales: y = x W^T,
// W[n][k] = code(n, k) * scale(n, k / group), and the gated form
// h = act(x Wg^T) * (x Wu^T).
//
// What must move is the weights, half a byte each and read once, so they go straight
// from global memory to registers, 16 bytes (32 codes of a row) a lane. A workgroup has
// 16 rows of W and all of K, its waves a part of K each; their sums meet in LDS. The
// 16x16x32 matrix instruction does the products for up to 16 tokens at a time whatever
// their number: its A operand is x (rows: tokens), its B operand the weights, whose column
// (a row of W) stays in the lane that loaded the codes, so that the lane's own scale
// multiplies its four sums. Codes become bfloat16 or float16 exactly (two a conversion
// instruction), sums over a group are float32, then scaled and added up in float32.
//
// A lane's 16 bytes are 32 k of one group of 32, but an instruction sums over the 8 k of each
// of four lanes: two exchanges between lane rows (permlane32_swap, permlane16_swap) first turn
// the 4 words of 4 lanes around, so that one instruction's 32 k are one group's.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "block.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

constexpr int kSpan = 128;  // k of a step: 32 of each of the four lanes of a row

#ifdef __HIP_DEVICE_COMPILE__
template <class T>
__device__ __forceinline__ typename T::vec8 decode8(uint32_t w);
template <>
__device__ __forceinline__ TypeBF16::vec8 decode8<TypeBF16>(uint32_t w) {
  TypeBF16::vec2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3)};
  return __builtin_bit_cast(TypeBF16::vec8, v);
}
template <>
__device__ __forceinline__ TypeF16::vec8 decode8<TypeF16>(uint32_t w) {
  TypeF16::vec2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3)};
  return __builtin_bit_cast(TypeF16::vec8, v);
}

// The codes of a lane for one step (32 of its row) and the scales of the step's groups.
template <int kScale, int kGroup>
struct Step {
  static constexpr int kScales = kSpan / kGroup;
  u32x4v codes;
  float scale[kScales];

  __device__ __forceinline__ void load(const W4Matrix& m, int64_t row, int64_t K, int64_t row_bytes,
                                       int64_t groups, int64_t step, int q, bool whole) {
    const uint8_t* c = m.codes + row * row_bytes + step * (kSpan / 2) + 16 * q;
    const int64_t g0 = row * groups + step * kScales;
    if (whole) {
      __builtin_memcpy(&codes, c, 16);
      if constexpr (kScale == HOBFLOPS_SCALE_POW2) {
        uint8_t s[kScales];
        __builtin_memcpy(s, (const uint8_t*)m.scales + g0, sizeof s);
#pragma unroll
        for (int i = 0; i < kScales; ++i) scale[i] = pow2_scale_of(s[i]);
      } else if constexpr (kScale == HOBFLOPS_SCALE_BF16) {
        uint16_t s[kScales];
        __builtin_memcpy(s, (const uint16_t*)m.scales + g0, sizeof s);
#pragma unroll
        for (int i = 0; i < kScales; ++i) scale[i] = __uint_as_float((uint32_t)s[i] << 16);
      } else {
        __builtin_memcpy(scale, (const float*)m.scales + g0, sizeof scale);
      }
    } else {  // the end of a row: no byte and no scale beyond it
      const int64_t first = step * (kSpan / 2) + 16 * q;
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (first + i < row_bytes) w[i >> 2] |= (uint32_t)c[i] << (8 * (i & 3));
#pragma unroll
      for (int i = 0; i < 4; ++i) codes[i] = w[i];
#pragma unroll
      for (int i = 0; i < kScales; ++i)
        scale[i] = step * kScales + i < groups ? load_scale(m.scales, g0 + i, kScale) : 0.0f;
    }
  }
  // word[m]: 8 codes of the step's 32 k from 32 m on
  __device__ __forceinline__ void words(uint32_t (&word)[4]) const {
    const auto a = __builtin_amdgcn_permlane32_swap(codes[0], codes[1], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(codes[2], codes[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    word[0] = c[0];
    word[1] = c[1];
    word[2] = d[0];
    word[3] = d[1];
  }
};

// 8 values of a token's row from k on; zeros beyond the row's end.
template <class T>
__device__ __forceinline__ typename T::vec8 load_x(const typename T::elem* row, int64_t k,
                                                   int64_t K, bool whole) {
  typename T::vec8 v;
  if (whole) {
    __builtin_memcpy(&v, row + k, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : (typename T::elem)0.0f;
  }
  return v;
}
#endif

// NT: groups of 16 tokens of a workgroup.
template <class T, int kScale, int kGroup, int NT, bool kGated>
__global__ __launch_bounds__(512) void w4_kernel(W4Product p) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename T::elem E;
  constexpr int kMats = kGated ? 2 : 1, U = NT == 1 ? 2 : 1, kPer = kGroup / 32;
  extern __shared__ __align__(16) uint8_t lds[];
  f32x4* sums = (f32x4*)lds;  // [wave][matrix][token group][lane]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int col = lane & 15, q = lane >> 4, turn = (q & 1) << 1 | q >> 1;
  const int64_t n = (int64_t)blockIdx.x * 16 + col, t0 = (int64_t)blockIdx.y * (16 * NT);
  const int64_t row = n < p.N ? n : p.N - 1;
  const int64_t row_bytes = (p.K + 1) / 2, groups = (p.K + kGroup - 1) / kGroup;
  const int64_t steps = (p.K + kSpan - 1) / kSpan, per = (steps + waves - 1) / waves;
  const int64_t first = wave * per, last = first + per < steps ? first + per : steps;
  f32x4 acc[kMats][NT] = {};

  const auto load_xs = [&](int64_t step, int m, int j, bool whole) {
    const int64_t t = t0 + 16 * j + col;
    typename T::vec8 v = {};
    if (t < p.T) v = load_x<T>((const E*)p.x + t * p.ldx, step * kSpan + 32 * m + 8 * turn, p.K, whole);
    return v;
  };
  const auto run = [&](int64_t step, auto count, bool whole) {
    constexpr int N = decltype(count)::value;
    Step<kScale, kGroup> s[N][kMats];
    typename T::vec8 x[N][4];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i][0].load(p.w, row, p.K, row_bytes, groups, step + i, q, whole);
      if constexpr (kGated) s[i][1].load(p.w_up, row, p.K, row_bytes, groups, step + i, q, whole);
    }
    if constexpr (NT == 1) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int m = 0; m < 4; ++m) x[i][m] = load_xs(step + i, m, 0, whole);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t word[kMats][4];
#pragma unroll
      for (int c = 0; c < kMats; ++c) s[i][c].words(word[c]);
      f32x4 part[kMats][NT];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        typename T::vec8 w[kMats];
#pragma unroll
        for (int c = 0; c < kMats; ++c) w[c] = decode8<T>(word[c][m]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const typename T::vec8 v = NT == 1 ? x[i][m] : load_xs(step + i, m, j, whole);
#pragma unroll
          for (int c = 0; c < kMats; ++c) {
            const f32x4 zero = {};
            part[c][j] = T::mfma(v, w[c], m % kPer == 0 ? zero : part[c][j]);
            if (m % kPer == kPer - 1) {
              const float f = s[i][c].scale[m / kPer];
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[c][j][r] += f * part[c][j][r];
            }
          }
        }
      }
    }
  };
  const int64_t whole = p.K / kSpan < last ? p.K / kSpan : last;  // steps before it are whole
  int64_t s = first;
  for (; s + U <= whole; s += U) run(s, std::integral_constant<int, U>(), true);
  for (; s < whole; ++s) run(s, std::integral_constant<int, 1>(), true);
  if (s < last) run(s, std::integral_constant<int, 1>(), false);

#pragma unroll
  for (int c = 0; c < kMats; ++c)
#pragma unroll
    for (int j = 0; j < NT; ++j) sums[((wave * kMats + c) * NT + j) * 64 + lane] = acc[c][j];
  __syncthreads();
  for (int j = wave; j < NT; j += waves) {
    f32x4 y[kMats] = {};
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int c = 0; c < kMats; ++c) y[c] += sums[((w * kMats + c) * NT + j) * 64 + lane];
    if (n < p.N) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t t = t0 + 16 * j + 4 * q + r;
        if (t >= p.T) continue;
        const float v = kGated ? gate_act(y[0][r], p.act) * y[kMats - 1][r] : y[0][r];
        ((E*)p.y)[t * p.ldy + n] = (E)v;
      }
    }
  }
#endif
}

template <class T, int kScale, int kGroup, int NT, bool kGated>
void launch_tiles(const W4Product& p, hipStream_t stream) {
  const int waves = 8;
  const dim3 grid((unsigned)((p.N + 15) / 16), (unsigned)((p.T + 16 * NT - 1) / (16 * NT)));
  w4_kernel<T, kScale, kGroup, NT, kGated>
      <<<grid, 64 * waves, waves * NT * (kGated ? 2 : 1) * 1024, stream>>>(p);
}
template <class T, int kScale, int kGroup>
void launch_tokens(const W4Product& p, hipStream_t stream) {
  if (p.w_up.codes)
    p.T <= 16 ? launch_tiles<T, kScale, kGroup, 1, true>(p, stream)
              : launch_tiles<T, kScale, kGroup, 4, true>(p, stream);
  else
    p.T <= 16 ? launch_tiles<T, kScale, kGroup, 1, false>(p, stream)
              : launch_tiles<T, kScale, kGroup, 4, false>(p, stream);
}
template <class T, int kScale>
void launch_group(const W4Product& p, hipStream_t stream) {
  if (p.group == 32) launch_tokens<T, kScale, 32>(p, stream);
  if (p.group == 64) launch_tokens<T, kScale, 64>(p, stream);
  if (p.group == 128) launch_tokens<T, kScale, 128>(p, stream);
}
template <class T>
void launch_scale(const W4Product& p, hipStream_t stream) {
  if (p.scale == HOBFLOPS_SCALE_POW2) launch_group<T, HOBFLOPS_SCALE_POW2>(p, stream);
  if (p.scale == HOBFLOPS_SCALE_BF16) launch_group<T, HOBFLOPS_SCALE_BF16>(p, stream);
  if (p.scale == HOBFLOPS_SCALE_F32) launch_group<T, HOBFLOPS_SCALE_F32>(p, stream);
}

}  // namespace

hipError_t launch_w4(const W4Product& all, hipStream_t stream) {
  // tokens in parts, for the grid's second axis
  constexpr int64_t kTokens = (int64_t)1 << 21;
  for (int64_t t = 0; t < all.T; t += kTokens) {
    W4Product p = all;
    p.T = all.T - t < kTokens ? all.T - t : kTokens;
    p.x = (const uint16_t*)all.x + t * all.ldx;
    p.y = (uint16_t*)all.y + t * all.ldy;
    if (p.type == HOBFLOPS_TYPE_BF16)
      launch_scale<TypeBF16>(p, stream);
    else
      launch_scale<TypeF16>(p, stream);
  }
  return hipGetLastError();
}

}  // namespace hobflops
