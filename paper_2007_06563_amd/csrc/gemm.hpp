// The matrix products of the gated block: 16-bit operands, float32 sums.
//
// A workgroup computes a tile of BI x BJ sums, D[i][j] = sum_k A[i][k] B[j][k], 64 of
// k at a time. The tiles of A and B go from global memory straight into LDS (buffer
// loads with the LDS as their target, 16 bytes a lane), into one of two stages while the
// matrix instructions work on the other. Two layouts of an operand in memory:
//  - K-contiguous ([row][k], the weights and x of the forward product): an LDS row is 64
//    k (128 bytes), and a fragment (8 k of a row a lane) is one 16-byte LDS read.
//  - K-major ([k][column], the weights of dx, both operands of the weight gradients): an
//    LDS row is the tile's columns of one k, and two transposing 8-byte LDS reads give a
//    fragment, so that no operand is transposed in memory.
// The 16-byte chunks of an LDS row are stored at a place that is XORed with bits of the row's
// number, and the lanes fetch from global memory accordingly (the target of a load
// into LDS is linear in the lane): the reads of a fragment then fall on different banks.
//
// Rows and k beyond an operand's end come back as zero from the buffer descriptor's
// range check (K-contiguous rows: lanes whose k is beyond the end are given an offset out
// of range), so that no element of a neighbouring row takes part in a sum. Operands have 16-byte
// aligned rows; the K of a K-contiguous one is a multiple of 8.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "narrow.hpp"

namespace hobflops {

constexpr int kStepK = 64;
constexpr uint32_t kOutOfRange = 0x80000000u;  // an offset beyond every descriptor's range

typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// The device code below uses types that the host compiler does not have; a kernel that
// uses it has an empty body there.
#ifdef __HIP_DEVICE_COMPILE__

// A descriptor of what is left of an operand from a point on: `left` bytes, at most 2^31.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rest_of(const void* p, int64_t left) {
  const int64_t n = left < 0 ? 0 : left > (int64_t)kOutOfRange ? (int64_t)kOutOfRange : left;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)n, 0x00020000);
}

// Loads a tile of R rows and 64 k of a K-contiguous operand (one or, split by rows into halves,
// two tensors) into a stage. NW waves.
template <int R, int NW, int kParts>
struct LoadRows {
  static constexpr int kLoads = R / 8 / NW;  // of a wave: 8 rows each
  const uint8_t* p[kParts];
  int64_t left[kParts];  // bytes from the tile's first row on
  int64_t k_left;
  uint32_t step, off, chunk;  // bytes between a wave's loads; the lane's offset; its first k / 8

  __device__ __forceinline__ void start(const void* const (&src)[kParts], int64_t ld, int64_t rows,
                                        int64_t row0, int64_t K, int64_t k0, int wave, int lane) {
    const int r = 8 * wave + (lane >> 3);
    chunk = (lane & 7) ^ ((r >> 1) & 7);
    off = (uint32_t)(r * ld * 2) + chunk * 16;
    step = (uint32_t)(8 * NW * ld * 2);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      p[i] = (const uint8_t*)src[i] + (row0 * ld + k0) * 2;
      left[i] = ((rows - row0 - 1) * ld + K - k0) * 2;
    }
    k_left = K - k0;
  }
  __device__ __forceinline__ void load(uint8_t* stage, int wave) {
    const uint32_t o = (int64_t)(chunk * 8) < k_left ? off : kOutOfRange;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int part = i * kParts / kLoads;
      const uint32_t so = (uint32_t)(i - part * kLoads / kParts) * step;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rest_of(p[part], left[part]),
                                               (lds_byte*)(stage + (wave + NW * i) * 1024), 16,
                                               o + so, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      p[i] += kStepK * 2;
      left[i] -= kStepK * 2;
    }
    k_left -= kStepK;
  }
};

// Loads a tile of 64 k and R columns of a K-major operand (one or, one after the other along k,
// two tensors) into a stage.
template <int R, int NW>
struct LoadColumns {
  static constexpr int kRowsPer = 512 / R;                 // k of a load
  static constexpr int kLoads = kStepK / kRowsPer / NW;    // of a wave
  const uint8_t* p;
  int64_t left, advance;
  uint32_t step, off;

  // part: the tensor's K rows from k0 on
  __device__ __forceinline__ void start(const void* src, int64_t ld, int64_t cols, int64_t col0,
                                        int64_t K, int64_t k0, int wave, int lane) {
    const int k = wave * kRowsPer + lane / (R / 8);
    const int f = (k & 3) | ((k >> 3) & 1) << 2;
    off = (uint32_t)(k * ld * 2) + (uint32_t)(((lane % (R / 8)) ^ (f << 1)) * 16);
    step = (uint32_t)(NW * kRowsPer * ld * 2);
    advance = kStepK * ld * 2;
    p = (const uint8_t*)src + (k0 * ld + col0) * 2;
    left = ((K - k0 - 1) * ld + cols - col0) * 2;
  }
  __device__ __forceinline__ void load(uint8_t* stage, int wave) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rest_of(p, left),
                                               (lds_byte*)(stage + (wave + NW * i) * 1024), 16,
                                               off + (uint32_t)i * step, 0, 0, 0);
    p += advance;
    left -= advance;
  }
};

// Fragments of a stage: N of 16 rows each, k step ks (32 k).
template <class T, int N>
struct ReadRows {
  uint32_t at;
  __device__ __forceinline__ void start(int row0, int lane) {
    const int r = lane & 15, q = lane >> 4;
    at = (uint32_t)((row0 + r) * 128 + ((q ^ (r >> 1)) << 4));
  }
  __device__ __forceinline__ typename T::vec8 get(const uint8_t* stage, int i, int ks) const {
    return *(const typename T::vec8*)(stage + (at ^ (uint32_t)(ks * 64)) + i * 2048);
  }
};
template <class T, int N, int R>
struct ReadColumns {
  uint32_t at[N];
  __device__ __forceinline__ void start(int col0, int lane) {
    const int r = lane & 15, q = lane >> 4;
    const int f = (r >> 2) | (q & 1) << 2;
    const uint32_t row = (uint32_t)((8 * q + (r >> 2)) * R * 2 + (r & 3) * 8);
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = row + (uint32_t)(((col0 / 16 + i) ^ f) << 5);
  }
  __device__ __forceinline__ typename T::vec8 get(const uint8_t* stage, int i, int ks) const {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint8_t* a = stage + at[i] + ks * 32 * R * 2;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 4 * R * 2));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename T::vec8, v);
  }
};

// Waits for a wave's loads into LDS, then for the other waves: their loads have landed too, and
// their reads of the stage that the next loads overwrite are done.
__device__ __forceinline__ void stage_ready() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

#endif  // __HIP_DEVICE_COMPILE__

// Tile of a workgroup: consecutive numbers go to the eight XCDs in turn, so that number b becomes
// tile b / 8 of XCD b % 8's range; within a range, tiles are taken in groups of 8 in i, so that the
// tiles that run at a time on an XCD share rows of A and of B in its L2.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t ni, uint32_t nj, uint32_t& ti,
                                        uint32_t& tj) {
  const uint32_t n = ni * nj, x = b & 7, each = n >> 3, more = n & 7;
  const uint32_t t = x * each + (x < more ? x : more) + (b >> 3);
  const uint32_t group = 8 * nj, g = t / group, in = t - g * group;
  const uint32_t height = ni - 8 * g < 8 ? ni - 8 * g : 8;
  ti = 8 * g + in % height;
  tj = in / height;
}

}  // namespace hobflops
