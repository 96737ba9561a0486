// Products of a few tokens with 4-bit weights under group scales: y = x W^T,
// W[n][k] = code(n, k) * scale(n, k / group), and the gated form
// h = act(x Wg^T) * (x Wu^T).
//
// What must move is the weights, half a byte each and read once: they go from global
// memory into LDS in whole lines, the next ones under way while some are multiplied. A wave has 16
// rows of W, all of K or a part; the sums of the parts meet in LDS. The
// 16x16x32 matrix instruction does the products for up to 16 tokens at a time whatever
// their number: its A operand is x (rows: tokens), its B operand the weights, whose column
// (a row of W) stays in one lane, so that the lane's own scale multiplies its four sums.
// Codes become bfloat16 or float16 exactly (two a conversion instruction), sums over a
// group are float32, then scaled and added up in float32.
//
// A lane's 16 bytes of an LDS read are 32 k of one group of 32, but an instruction sums over the 8 k of each
// of four lanes: two exchanges between lane rows (permlane32_swap, permlane16_swap) first turn
// the 4 words of 4 lanes around, so that one instruction's 32 k are one group's.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "block.hpp"
#include "narrow.hpp"

namespace hobflops {
namespace {

constexpr int kUnit = 256;   // k of a unit: two times 32 of each of the four lanes of a row
constexpr int kWaves = 8;    // of a workgroup of w4_kernel
constexpr int kStreamUnits = 2;  // of a wave, at most, in the streaming kernel: their scales are in registers
constexpr int kCUs = 256;
constexpr int kLds = 160 * 1024;

#ifdef __HIP_DEVICE_COMPILE__
// Eight codes times a power of two.
template <class T>
__device__ __forceinline__ typename T::vec8 decode8(uint32_t w, float s);
template <>
__device__ __forceinline__ TypeBF16::vec8 decode8<TypeBF16>(uint32_t w, float s) {
  TypeBF16::vec2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)};
  return __builtin_bit_cast(TypeBF16::vec8, v);
}
template <>
__device__ __forceinline__ TypeF16::vec8 decode8<TypeF16>(uint32_t w, float s) {
  TypeF16::vec2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3)};
  return __builtin_bit_cast(TypeF16::vec8, v);
}

// Whether all four bytes are scales 2^k with which the weights themselves, code times 2^k, are exact in the
// type: k of -63..64 in bfloat16, -19..12 in float16 (0.5 * 2^-19 is one of its subnormal values).
template <class T>
__device__ __forceinline__ bool exact_scales(uint32_t w) {
  if constexpr (std::is_same_v<T, TypeBF16>)
    return ((w ^ (w << 1)) & 0x80808080u) == 0x80808080u;
  else
    return ((w + 0x14141414u) & 0xE0E0E0E0u) == 0x80808080u;
}

// A bfloat16 x may be so large, from 2^117 on, that a sum of it times bare codes leaves float32's range where the
// formula's terms, with a small scale, are far within. So a scale is taken in two factors: a power of two with
// which the weights are exact (its own, or the nearest of exact_scales), which goes into them, and the
// rest, which multiplies a group's sum. (Four instructions a scale. One token, both projections of 4096 -> 11264
// in groups of 32: 15.7 us with bfloat16 x, 14.7 with float16, whose sums with bare codes do not come near 2^128.)
template <class T>
constexpr bool kWide = std::is_same_v<T, TypeBF16>;
struct ScaleParts {
  float inside, rest;
};
template <bool kSplit>
__device__ __forceinline__ ScaleParts parts_of(float s) {
  if constexpr (!kSplit) return {1.0f, s};
  constexpr uint32_t lo = 64u << 23, hi = 191u << 23;
  uint32_t e = __float_as_uint(s) & 0x7F800000u;
  e = e < lo ? lo : e > hi ? hi : e;
  return {__uint_as_float(e), s * __uint_as_float((254u << 23) - e)};
}

// The scales of a row's groups of a unit (256 k, or kSpan), as they are in memory until they are used: a
// conversion next to the load would wait for it.
template <int kScale, int kGroup, int kSpan = kUnit>
struct Scales {
  static constexpr int kCount = kSpan / kGroup;
  static constexpr int kBytes = kScale == HOBFLOPS_SCALE_POW2 ? 1 : kScale == HOBFLOPS_SCALE_BF16 ? 2 : 4;
  static constexpr int kWords = (kCount * kBytes + 3) / 4;
  uint32_t word[kWords];
  int left;  // groups of the row from the first on; those beyond count as zero, their codes meet zeros of x
  __device__ __forceinline__ void load(const void* scales, int64_t row, int groups, int unit, int64_t N) {
    const int g0 = unit * kCount;
    left = groups - g0;
    const int64_t at = row * groups + g0;
    const uint8_t* p = (const uint8_t*)scales + at * kBytes;
    if (at + kCount <= N * groups) {  // beyond a row's end there are the next row's
      word[kWords - 1] = 0;
      __builtin_memcpy(word, p, kCount * kBytes);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) word[i] = 0;
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (at + i < N * groups) {
          uint32_t v = 0;
          __builtin_memcpy(&v, p + i * kBytes, kBytes);
          word[i * kBytes / 4] |= v << (8 * (i * kBytes & 3));
        }
    }
  }
  // whether the scales can go into the weights (bytes that only fill the last word count as 1)
  template <class T>
  __device__ __forceinline__ bool exact() const {
    bool all = kScale == HOBFLOPS_SCALE_POW2;
#pragma unroll
    for (int i = 0; i < kWords; ++i)
      all = all && exact_scales<T>(kCount == 1   ? word[i] | 0x7F7F7F00u
                                   : kCount == 2 ? word[i] | 0x7F7F0000u
                                                 : word[i]);
    return all;
  }
  __device__ __forceinline__ float exact_get(int i) const {
    const int at = i / (kGroup / 32);
    return __uint_as_float((word[at / 4] >> (8 * (at & 3)) & 255u) << 23);
  }
  // of the 32 k from 32 i on
  __device__ __forceinline__ float get(int i) const {
    const int g = i / (kGroup / 32), at = g * kBytes;
    const uint32_t w = word[at / 4] >> (8 * (at & 3));
    float f = __uint_as_float(w);
    if constexpr (kScale == HOBFLOPS_SCALE_POW2) f = pow2_scale_of(w & 255u);
    if constexpr (kScale == HOBFLOPS_SCALE_BF16) f = __uint_as_float(w << 16);
    return g < left ? f : 0.0f;
  }
};

// Of the codes of a step that the four lanes of a row hold, 32 each: word[m] is this lane's 8 of those
// from 32 m on.
__device__ __forceinline__ void turn_codes(u32x4v codes, uint32_t (&word)[4]) {
  const auto a = __builtin_amdgcn_permlane32_swap(codes[0], codes[1], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(codes[2], codes[3], false, false);
  const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  word[0] = c[0];
  word[1] = c[1];
  word[2] = d[0];
  word[3] = d[1];
}

#endif

#ifdef __HIP_DEVICE_COMPILE__
// A unit's products: codes[c] its 16 rows of 128 bytes in LDS, x(i) the x of the 32 k from 32 i on.
// Scales that are exact powers of two go into the weights, whose products then sum up in place; others
// multiply the sums of a group.
template <class T, int kScale, int kGroup, int kMats, class X>
__device__ __forceinline__ void multiply_unit(const uint8_t* const (&codes)[kMats],
                                              const Scales<kScale, kGroup> (&scale)[kMats], int lane,
                                              X x, f32x4 (&acc)[kMats]) {
  typedef typename T::vec8 Vec;
  constexpr int kPer = kGroup / 32;
  const int col = lane & 15, q = lane >> 4;
  bool exact = true;
#pragma unroll
  for (int c = 0; c < kMats; ++c) exact = exact && scale[c].template exact<T>();
  const bool inside = kScale == HOBFLOPS_SCALE_POW2 && __all(exact);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t word[kMats][4];
#pragma unroll
    for (int c = 0; c < kMats; ++c)
      turn_codes(*(const u32x4v*)(codes[c] + col * 128 + (((4 * h + q) ^ (col >> 1)) << 4)), word[c]);
    if (inside) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const Vec v = x(4 * h + m);
#pragma unroll
        for (int c = 0; c < kMats; ++c)
          acc[c] = T::mfma(v, decode8<T>(word[c][m], scale[c].exact_get(4 * h + m)), acc[c]);
      }
    } else {
      f32x4 sum[kMats];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const Vec v = x(4 * h + m);
#pragma unroll
        for (int c = 0; c < kMats; ++c) {
          const f32x4 zero = {};
          const ScaleParts f = parts_of<kWide<T>>(scale[c].get(4 * h + m));
          sum[c] = T::mfma(v, decode8<T>(word[c][m], f.inside), m % kPer == 0 ? zero : sum[c]);
          if (m % kPer == kPer - 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[c][r] += f.rest * sum[c][r];
          }
        }
      }
    }
  }
}

// A load into LDS, 16 bytes a lane, at `lds` on; zeros from offsets out of the descriptor's range. These are
// assembly since the compiler, which knows what a load into LDS is, would wait for all of them
// before each read of LDS; loaded() is the wait. M0 is the target's place.
__device__ __forceinline__ void load_lds(u32x4v rows, uint32_t off, const uint8_t* to) {
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)to;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(rows)
               : "memory", "m0");
}
__device__ __forceinline__ void loaded() {
  __builtin_amdgcn_s_waitcnt(0x0070);  // no load and no LDS read under way; the compiler counts this one
  asm volatile("" ::: "memory");
}
// Before a load into LDS that was just read.
__device__ __forceinline__ void reads_done() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}
// The descriptor of `bytes` of raw 32-bit data.
__device__ __forceinline__ u32x4v raw_rows(const void* p, uint32_t bytes) {
  const uint64_t at = (uint64_t)(uintptr_t)p;
  return u32x4v{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
}

// Loads of a tile's codes: 16 rows of 128 bytes a unit and matrix. The 16-byte chunks of a row stand at a
// place XORed with bits of the row's number, so that a read of 16 rows falls on different banks.
template <int kMats>
struct CodeLoads {
  u32x4v rows[kMats];
  uint32_t off[2];
  __device__ __forceinline__ void start(const W4Product& p, int64_t tile, int row_bytes, int lane) {
    const int left = (int)(p.N - tile * 16 < 16 ? p.N - tile * 16 : 16);
#pragma unroll
    for (int c = 0; c < kMats; ++c)
      rows[c] = raw_rows((c ? p.w_up : p.w).codes + tile * 16 * row_bytes, (uint32_t)(left * row_bytes));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 8 * i + (lane >> 3);
      off[i] = (uint32_t)(r * row_bytes + (((lane & 7) ^ (r >> 1)) << 4));
    }
  }
  __device__ __forceinline__ void fetch(int unit, const uint8_t* slot) const {
#pragma unroll
    for (int c = 0; c < kMats; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        load_lds(rows[c], off[h] + (uint32_t)unit * 128, slot + c * 2048 + h * 1024);
  }
};

// Loads of x, a unit (512 bytes) of two tokens at a time, the chunks' places XORed with the token's number.
struct XLoads {
  u32x4v rows;
  uint32_t ld2;
  int tokens, K;
  __device__ __forceinline__ void start(const W4Product& p, int64_t t0) {
    tokens = (int)(p.T - t0 < 16 ? p.T - t0 : 16);
    K = (int)p.K;
    ld2 = (uint32_t)(p.ldx * 2);
    rows = raw_rows((const uint8_t*)p.x + t0 * p.ldx * 2, (uint32_t)(tokens - 1) * ld2 + (uint32_t)K * 2);
  }
  __device__ __forceinline__ void fetch(int token, int unit, int lane, const uint8_t* to) const {
    const int k = unit * kUnit + ((lane & 31) ^ (token & 15)) * 8;
    const bool in = token < tokens && k < K;
    load_lds(rows, in ? (uint32_t)token * ld2 + (uint32_t)k * 2 : 0x80000000u, to);
  }
};

// Output of 16 rows for 16 tokens: y the sums of a lane's column, its tokens 4 (lane / 16) + 0..3.
template <class T, int kMats>
__device__ __forceinline__ void store_tokens(const W4Product& p, int64_t n, int64_t t0, int lane,
                                             const f32x4 (&y)[kMats]) {
  if (n >= p.N) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t t = t0 + 4 * (lane >> 4) + r;
    if (t >= p.T) continue;
    const float v = kMats > 1 ? gate_act(y[0][r], p.act) * y[kMats - 1][r] : y[0][r];
    ((typename T::elem*)p.y)[t * p.ldy + n] = (typename T::elem)v;
  }
}
#endif

// A workgroup's waves have a part of K each, in units of 256 k (128 bytes of a row: a whole cache
// line). Codes and x go into LDS first: loads into it can take 128 bytes of each of 8 rows, where registers
// would need 64 of 16 (the column of the matrix instruction is the lane), and hold no registers while they
// are under way. A workgroup has up to 16 tokens, those of neighbouring numbers the same tiles' other tokens.

// The part of K of a wave.
__device__ __forceinline__ int part_of(int units, int wave, int waves) { return units * wave / waves; }

// x of all K fits LDS: as many workgroups as run at a time, each with the tiles (16 rows) that are
// `stride` apart. x is loaded once; a tile's codes and scales are under way while the tile before is
// multiplied.
// Bound by HBM and, in short calls, by latency: 5 x 4104 -> 50257 in 36 us, 3.2 TB/s of codes, scales and y; one token,
// both projections of 4096 -> 11264, 12.6 us, 3.9 TB/s; 4096 -> 4096 in 5.8 us, mostly a
// launch and the loads' latency. With codes from global memory to registers (16 lines of 16 bytes a load) the
// first two took 47 and 14.5 us.
template <class T, int kScale, int kGroup, bool kGated>
__global__ __launch_bounds__(1024) void w4_stream_kernel(W4Product p, int parts, int stride) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename T::vec8 Vec;
  typedef Scales<kScale, kGroup> Sc;
  constexpr int kMats = kGated ? 2 : 1, kSlot = kMats * 2048;
  extern __shared__ __align__(1024) uint8_t lds[];  // two sets of sums, two of the units, x
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int col = lane & 15, q = lane >> 4, turn = (q & 1) << 1 | q >> 1;
  const int K = (int)p.K, row_bytes = K / 2, groups = (K + kGroup - 1) / kGroup;
  const int units = (K + kUnit - 1) / kUnit;
  const int first = part_of(units, wave, waves), count = part_of(units, wave + 1, waves) - first;
  const int64_t t0 = (int64_t)(blockIdx.x % parts) * 16;
  XLoads x;
  x.start(p, t0);
  const int tokens = x.tokens, lanes = (tokens + 3) / 4 * 16;  // that hold sums of tokens
  const int sum_bytes = waves * kMats * lanes * 16;
  uint8_t* const sums0 = lds + 2 * units * kSlot;
  uint8_t* const xs = sums0 + 2 * sum_bytes;
  const uint32_t tiles = (uint32_t)((p.N + 15) / 16);
  const auto fetch = [&](uint32_t tile, int set, Sc(&s)[kStreamUnits][kMats]) {
    CodeLoads<kMats> loads;
    loads.start(p, tile, row_bytes, lane);
    const int64_t n = (int64_t)tile * 16 + col, row = n < p.N ? n : p.N - 1;
#pragma unroll
    for (int i = 0; i < kStreamUnits; ++i)
      if (i < count) {
        loads.fetch(first + i, lds + (set * units + first + i) * kSlot);
        s[i][0].load(p.w.scales, row, groups, first + i, p.N);
        if constexpr (kGated) s[i][1].load(p.w_up.scales, row, groups, first + i, p.N);
      }
  };
  Sc now[kStreamUnits][kMats], next[kStreamUnits][kMats];
  uint32_t tile = blockIdx.x / parts;
  fetch(tile, 0, now);
  for (int i = 2 * wave; i < tokens * units; i += 2 * waves) {
    const int pair = i + (lane >> 5);
    x.fetch(pair / units, pair % units, lane, xs + i * 512);
  }
  loaded();
  __syncthreads();
  const int t = col < tokens ? col : tokens - 1;  // tokens beyond the last are computed and not stored
  const uint8_t* const x_of = xs + t * units * 512;
  for (int n = 0; tile < tiles; ++n) {
    const int set = n & 1;
    loaded();
    const uint32_t after = tile + stride;
    if (after < tiles) fetch(after, set ^ 1, next);
    f32x4 acc[kMats] = {};
#pragma unroll
    for (int i = 0; i < kStreamUnits; ++i)
      if (i < count) {
        const uint8_t* const s = lds + (set * units + first + i) * kSlot;
        const uint8_t* codes[kMats];
#pragma unroll
        for (int c = 0; c < kMats; ++c) codes[c] = s + c * 2048;
        const int k8 = (first + i) * (kUnit / 8) + turn;
        multiply_unit<T, kScale, kGroup, kMats>(
            codes, now[i], lane, [&](int m) { return *(const Vec*)(x_of + (((k8 + 4 * m) ^ t) << 4)); }, acc);
      }
    // The waves' sums meet in LDS, one wave after the other adds a tile's. The set is written again
    // two tiles on, after a barrier that this tile's adding wave has reached, too.
    uint8_t* const sums = sums0 + set * sum_bytes;
    if (lane < lanes) {
#pragma unroll
      for (int c = 0; c < kMats; ++c) *(f32x4*)(sums + ((wave * kMats + c) * lanes + lane) * 16) = acc[c];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (wave == n % waves && lane < lanes) {
      f32x4 y[kMats] = {};
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int c = 0; c < kMats; ++c) y[c] += *(const f32x4*)(sums + ((w * kMats + c) * lanes + lane) * 16);
      store_tokens<T, kMats>(p, (int64_t)tile * 16 + col, t0, lane, y);
    }
#pragma unroll
    for (int i = 0; i < kStreamUnits; ++i)
#pragma unroll
      for (int c = 0; c < kMats; ++c) now[i][c] = next[i][c];
    tile = after;
  }
#endif
}

// An x that does not fit: a workgroup of eight waves a tile. The codes of up to `ring` units of a wave are
// under way at a time; x comes a unit at a time, a unit ahead where LDS has two places for it.
// 16 x 11264 -> 4096 in 13.0 us, 1.9 TB/s: a workgroup a CU and one tile each, so start and end count in full, and
// each reads all of x, four times the bytes of its codes, from L2.
template <class T, int kScale, int kGroup, bool kGated>
__global__ __launch_bounds__(512) void w4_kernel(W4Product p, int parts, int ring, int places) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename T::vec8 Vec;
  typedef Scales<kScale, kGroup> Sc;
  constexpr int kMats = kGated ? 2 : 1, kSlot = kMats * 2048;
  extern __shared__ __align__(1024) uint8_t lds[];  // of each wave: its units' codes, x
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, q = lane >> 4, turn = (q & 1) << 1 | q >> 1;
  const uint32_t tile = blockIdx.x / parts;
  const int64_t t0 = (int64_t)(blockIdx.x % parts) * 16;
  const int64_t n = (int64_t)tile * 16 + col, row = n < p.N ? n : p.N - 1;
  const int K = (int)p.K, row_bytes = K / 2, groups = (K + kGroup - 1) / kGroup;
  const int units = (K + kUnit - 1) / kUnit;
  const int first = part_of(units, wave, kWaves), last = part_of(units, wave + 1, kWaves);
  XLoads x;
  x.start(p, t0);
  const int pairs = (x.tokens + 1) / 2, each = ring * kSlot + places * pairs * 1024;
  uint8_t* const mine = lds + wave * each;
  uint8_t* const xs = mine + ring * kSlot;
  CodeLoads<kMats> loads;
  loads.start(p, tile, row_bytes, lane);
  const int t = col < x.tokens ? col : x.tokens - 1;  // tokens beyond the last are not stored
  const auto ahead = [&](int unit, Sc(&s)[kMats]) {
    for (int i = 0; i < pairs; ++i)
      x.fetch(2 * i + (lane >> 5), unit, lane, xs + ((unit % places) * pairs + i) * 1024);
    s[0].load(p.w.scales, row, groups, unit, p.N);
    if constexpr (kGated) s[1].load(p.w_up.scales, row, groups, unit, p.N);
  };
  f32x4 acc[kMats] = {};
  const auto multiply = [&](int unit, int slot, const Sc(&s)[kMats]) {
    const uint8_t* codes[kMats];
#pragma unroll
    for (int c = 0; c < kMats; ++c) codes[c] = mine + slot * kSlot + c * 2048;
    const uint8_t* const x_of = xs + (unit % places) * pairs * 1024 + t * 512;
    multiply_unit<T, kScale, kGroup, kMats>(
        codes, s, lane, [&](int m) { return *(const Vec*)(x_of + (((4 * m + turn) ^ t) << 4)); }, acc);
  };
  for (int begin = first; begin < last; begin += ring) {
    const int end = begin + ring < last ? begin + ring : last;
    reads_done();
    for (int u = begin; u < end; ++u) loads.fetch(u, mine + (u - begin) * kSlot);
    Sc now[kMats], next[kMats];
    ahead(begin, now);
    for (int u = begin; u < end; ++u) {
      loaded();
      if (places > 1 && u + 1 < end) ahead(u + 1, next);
      multiply(u, u - begin, now);
      if (places == 1 && u + 1 < end) {
        reads_done();
        ahead(u + 1, next);
      }
#pragma unroll
      for (int c = 0; c < kMats; ++c) now[c] = next[c];
    }
  }
  // the waves' sums, each where its codes were
#pragma unroll
  for (int c = 0; c < kMats; ++c) *(f32x4*)(mine + (c * 64 + lane) * 16) = acc[c];
  __syncthreads();
  if (wave == 0) {
    f32x4 y[kMats] = {};
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
      for (int c = 0; c < kMats; ++c) y[c] += *(const f32x4*)(lds + w * each + (c * 64 + lane) * 16);
    store_tokens<T, kMats>(p, n, t0, lane, y);
  }
#endif
}

// Many tokens: a tile of 64 rows and 64 tokens a workgroup, all of K, 128 at a time through three
// stages of LDS. A wave has 16 rows for all the tokens, so that a code is converted once for 64.
// Bound by the conversions and the matrix instructions of a wave, one after the other: 64 tokens, both
// projections of 8192 -> 16384, 61 us, 0.56 PFLOP/s.
constexpr int kStep = 128, kTileTokens = 64, kTileWaves = 4;
// Two workgroups on a CU where the registers for groups' sums and scales allow it.
template <int kScale, int kGroup, bool kGated>
constexpr int kTilesOnCU = kScale == HOBFLOPS_SCALE_POW2 || kGroup == 128 || (kGroup == 64 && !kGated) ? 2 : 1;
template <class T, int kScale, int kGroup, bool kGated>
__global__ __launch_bounds__(64 * kTileWaves, (kTilesOnCU<kScale, kGroup, kGated>)) void w4_tile_kernel(W4Product p) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename T::vec8 Vec;
  typedef Scales<kScale, kGroup, kStep> Sc;
  constexpr int kMats = kGated ? 2 : 1, NT = kTileTokens / 16, kPer = kGroup / 32, W = kTileWaves, S = 3;
  constexpr int kX = kTileTokens * kStep * 2, kXLoads = kX / 1024 / W, kCodes = kMats * 1024;
  // An array a stage, so that the compiler knows that loads into one do not touch the others, counts
  // them and waits for no more than the scales it needs.
  __shared__ __align__(1024) uint8_t x0[kX], x1[kX], x2[kX], c0[W * kCodes], c1[W * kCodes], c2[W * kCodes];
  uint8_t* const xs[3] = {x0, x1, x2};
  uint8_t* const cs[3] = {c0, c1, c2};
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, q = lane >> 4, turn = (q & 1) << 1 | q >> 1;
  const int64_t n0 = ((int64_t)blockIdx.x * W + wave) * 16, n = n0 + col, row = n < p.N ? n : p.N - 1;
  const int64_t t0 = (int64_t)blockIdx.y * kTileTokens;
  const int K = (int)p.K, row_bytes = K / 2, groups = (K + kGroup - 1) / kGroup;
  const int tokens = (int)(p.T - t0 < kTileTokens ? p.T - t0 : kTileTokens);
  const int left = (int)(p.N - n0 < 0 ? 0 : p.N - n0 < 16 ? p.N - n0 : 16);
  typedef __attribute__((address_space(3))) uint8_t lds_byte;
  const auto raw = [](const void* at, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(at), 0, (int)bytes, 0x00020000);
  };
  __amdgpu_buffer_rsrc_t rows[kMats];
#pragma unroll
  for (int c = 0; c < kMats; ++c)  // no rows: an empty range, all zeros
    rows[c] = raw((c ? p.w_up : p.w).codes + (left ? n0 : 0) * row_bytes, (uint32_t)(left * row_bytes));
  const uint32_t code_off = (uint32_t)((lane >> 2) * row_bytes + (((lane & 3) ^ (-(lane >> 4) & 3)) << 4));
  const uint32_t ld2 = (uint32_t)(p.ldx * 2);
  const auto x_rows = raw((const uint8_t*)p.x + t0 * p.ldx * 2, (uint32_t)(tokens - 1) * ld2 + (uint32_t)K * 2);
  Sc scale[S][kMats];
  const auto load = [&](int step, int stage, Sc(&s)[kMats]) {
    s[0].load(p.w.scales, row, groups, step, p.N);
    if constexpr (kGated) s[1].load(p.w_up.scales, row, groups, step, p.N);
#pragma unroll
    for (int c = 0; c < kMats; ++c)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rows[c], (lds_byte*)(cs[stage] + wave * kCodes + c * 1024), 16,
                                               code_off + (uint32_t)step * (kStep / 2), 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {  // four tokens of 256 bytes
      const int t = 4 * (wave * kXLoads + i) + (lane >> 4), k = step * kStep + ((lane & 15) ^ (t & 15)) * 8;
      const bool in = t < tokens && k < K;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rows, (lds_byte*)(xs[stage] + (wave * kXLoads + i) * 1024), 16,
                                               in ? (uint32_t)t * ld2 + (uint32_t)k * 2 : 0x80000000u, 0, 0, 0);
    }
  };
  f32x4 acc[kMats][NT];
  const auto multiply = [&](auto split, int stage, const Sc(&s)[kMats]) {
    uint32_t word[kMats][4];
    bool exact = true;
#pragma unroll
    for (int c = 0; c < kMats; ++c) {
      turn_codes(*(const u32x4v*)(cs[stage] + wave * kCodes + c * 1024 + col * 64 +
                                  ((q ^ (-(col >> 2) & 3)) << 4)),
                 word[c]);
      exact = exact && s[c].template exact<T>();
    }
    const auto x = [&](int m, int j) {
      return *(const Vec*)(xs[stage] + (16 * j + col) * 256 + (((4 * m + turn) ^ col) << 4));
    };
    if (kScale == HOBFLOPS_SCALE_POW2 && __all(exact)) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        Vec w[kMats];
#pragma unroll
        for (int c = 0; c < kMats; ++c) w[c] = decode8<T>(word[c][m], s[c].exact_get(m));
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const Vec v = x(m, j);
#pragma unroll
          for (int c = 0; c < kMats; ++c) acc[c][j] = T::mfma(v, w[c], acc[c][j]);
        }
      }
    } else {
      f32x4 sum[kMats][NT];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        Vec w[kMats];
        ScaleParts f[kMats];
#pragma unroll
        for (int c = 0; c < kMats; ++c) {
          f[c] = parts_of<decltype(split)::value>(s[c].get(m));
          w[c] = decode8<T>(word[c][m], f[c].inside);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const Vec v = x(m, j);
#pragma unroll
          for (int c = 0; c < kMats; ++c) {
            const f32x4 zero = {};
            sum[c][j] = T::mfma(v, w[c], m % kPer == 0 ? zero : sum[c][j]);
          }
        }
        if (m % kPer == kPer - 1) {
#pragma unroll
          for (int c = 0; c < kMats; ++c)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[c][j][r] += f[c].rest * sum[c][j][r];
        }
      }
    }
  };
  // A step's loads are issued S - 1 steps ahead, into the stage that all waves have read when the barrier is
  // passed. Its wait counts the loads into LDS alone; the scales' loads between them only make it
  // stricter. Steps beyond the last are of zeros.
  const int steps = (K + kStep - 1) / kStep;
  const auto sum_up = [&](auto split) {
#pragma unroll
    for (int c = 0; c < kMats; ++c)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[c][j] = f32x4{};
#pragma unroll
    for (int i = 0; i < S - 1; ++i) load(i, i, scale[i]);
    for (int k = 0; k < steps; k += S) {
#pragma unroll
      for (int i = 0; i < S; ++i) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * (kMats + kXLoads))
                     : "memory");
        load(k + i + S - 1, (i + S - 1) % S, scale[(i + S - 1) % S]);
        multiply(split, i, scale[i]);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // LDS becomes another workgroup's, or these sums' again
  };
  sum_up(std::false_type());
  if constexpr (kWide<T>) {
    // The scales in two factors only where a sum is not finite, all of it again: in every sum they would cost
    // more here (64 tokens, both projections of 8192 -> 16384 in groups of 32: 111 us, not 100).
    float z = 0.0f;
#pragma unroll
    for (int c = 0; c < kMats; ++c)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) z = __builtin_fmaf(acc[c][j][r], 0.0f, z);
    if (__syncthreads_or(z != z)) sum_up(std::true_type());
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    f32x4 y[kMats];
#pragma unroll
    for (int c = 0; c < kMats; ++c) y[c] = acc[c][j];
    store_tokens<T, kMats>(p, n, t0 + 16 * j, lane, y);
  }
#endif
}

// Any K and alignment, byte by byte: a wave a row of W and token. Bound by its instructions, a few a code.
template <class T>
__global__ __launch_bounds__(256) void w4_bytes_kernel(W4Product p) {
  typedef typename T::elem E;
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y;
  if (n >= p.N) return;
  const int64_t groups = (p.K + p.group - 1) / p.group;
  float sum[2] = {0.0f, 0.0f};
  for (int w = 0; w < (p.w_up.codes ? 2 : 1); ++w) {
    const W4Matrix& m = w ? p.w_up : p.w;
    for (int64_t k = lane; k < p.K; k += 64) {
      const uint32_t c = m.codes[n * ((p.K + 1) / 2) + k / 2] >> (4 * (k & 1));
      sum[w] += (float)((const E*)p.x)[t * p.ldx + k] *
                (decode_e2m1(c) * load_scale(m.scales, n * groups + k / p.group, p.scale));
    }
    for (int o = 32; o; o >>= 1) sum[w] += __shfl_xor(sum[w], o);
  }
  if (lane == 0)
    ((E*)p.y)[t * p.ldy + n] = (E)(p.w_up.codes ? gate_act(sum[0], p.act) * sum[1] : sum[0]);
}

template <class T, int kScale, int kGroup, bool kGated>
void launch_tiles(const W4Product& p, hipStream_t stream) {
  constexpr int kMats = kGated ? 2 : 1, kSlot = kMats * 2048;  // LDS of a unit
  const int64_t tiles = (p.N + 15) / 16, parts = (p.T + 15) / 16;
  const int units = (int)((p.K + kUnit - 1) / kUnit), tokens = (int)(p.T < 16 ? p.T : 16);
  // Tokens in tiles of 64 where that leaves a workgroup for half of the CUs: 64 tokens, both projections of
  // 8192 -> 16384: 61 us against 236 in tokens of 16; with 64 workgroups (4096 -> 4096) 22.6 against 19.4.
  const int64_t many = (p.T + kTileTokens - 1) / kTileTokens, rows = (p.N + 16 * kTileWaves - 1) / (16 * kTileWaves);
  if (p.T > 16 && rows * many >= kCUs / 2) {
    w4_tile_kernel<T, kScale, kGroup, kGated>
        <<<dim3((unsigned)rows, (unsigned)many), 64 * kTileWaves, 0, stream>>>(p);
    return;
  }
  {
    // the fewest units a wave that 16 waves make possible, and as few waves as that needs
    const int each = (units + 15) / 16, waves = (units + each - 1) / each;
    const int64_t bytes = (int64_t)2 * units * kSlot + 2 * waves * kMats * ((tokens + 3) / 4) * 256 +
                          ((int64_t)tokens * units + 1) * 512;
    if (each <= kStreamUnits && bytes <= kLds) {
      const int64_t run = kCUs * (bytes <= kLds / 2 && waves <= 8 ? 2 : 1);  // workgroups at a time
      int64_t stride = run / parts < 1 ? 1 : run / parts;
      if (stride > tiles) stride = tiles;
      w4_stream_kernel<T, kScale, kGroup, kGated>
          <<<(unsigned)(stride * parts), 64 * waves, (unsigned)bytes, stream>>>(p, (int)parts, (int)stride);
      return;
    }
  }
  const int each = (units + kWaves - 1) / kWaves, x = (tokens + 1) / 2 * 1024;
  // As many units under way as fit, and a second place for x only beside all of them. Two workgroups a
  // CU where there are enough of them and half of LDS still has three units, or all.
  const int half = kLds / 2 / kWaves, some = each < 3 ? each : 3;
  const int wave = tiles * parts > kCUs && (half - x) / kSlot >= some ? half : kLds / kWaves;
  const int places = (wave - 2 * x) / kSlot >= each ? 2 : 1;
  int ring = (wave - places * x) / kSlot;
  if (ring > each) ring = each;
  w4_kernel<T, kScale, kGroup, kGated>
      <<<(unsigned)(tiles * parts), 64 * kWaves, (unsigned)(kWaves * (ring * kSlot + places * x)), stream>>>(
          p, (int)parts, ring, places);
}
template <class T, int kScale, int kGroup>
void launch_mats(const W4Product& p, hipStream_t stream) {
  p.w_up.codes ? launch_tiles<T, kScale, kGroup, true>(p, stream)
               : launch_tiles<T, kScale, kGroup, false>(p, stream);
}
template <class T, int kScale>
void launch_group(const W4Product& p, hipStream_t stream) {
  if (p.group == 32) launch_mats<T, kScale, 32>(p, stream);
  if (p.group == 64) launch_mats<T, kScale, 64>(p, stream);
  if (p.group == 128) launch_mats<T, kScale, 128>(p, stream);
}
template <class T>
void launch_scale(const W4Product& p, hipStream_t stream) {
  // rows of codes and of x 4-byte aligned, 16 of x less than 2^31 bytes apart (of codes they are, K is at
  // most 2^24); fewer than 2^31 workgroups
  const bool words = p.K % 8 == 0 && ((uintptr_t)p.w.codes & 3u) == 0 && ((uintptr_t)p.w_up.codes & 3u) == 0 &&
                     ((uintptr_t)p.x & 3u) == 0 && p.ldx % 2 == 0 && p.ldx < (int64_t)1 << 26;
  if (!words) {
    w4_bytes_kernel<T><<<dim3((unsigned)((p.N + 3) / 4), (unsigned)p.T), 256, 0, stream>>>(p);
    return;
  }
  if (p.scale == HOBFLOPS_SCALE_POW2) launch_group<T, HOBFLOPS_SCALE_POW2>(p, stream);
  if (p.scale == HOBFLOPS_SCALE_BF16) launch_group<T, HOBFLOPS_SCALE_BF16>(p, stream);
  if (p.scale == HOBFLOPS_SCALE_F32) launch_group<T, HOBFLOPS_SCALE_F32>(p, stream);
}

}  // namespace

hipError_t launch_w4(const W4Product& all, hipStream_t stream) {
  // tokens in parts, for the grid's second axis; where 64 of x may be 2^31 bytes apart, in single tiles of 16
  const int64_t tokens = all.ldx < (int64_t)1 << 24 ? 4096 : 16;
  for (int64_t t = 0; t < all.T; t += tokens) {
    W4Product p = all;
    p.T = all.T - t < tokens ? all.T - t : tokens;
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
