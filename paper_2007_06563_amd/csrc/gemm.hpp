// The matrix products of the gated block: 16-bit operands, float32 sums.
//
// A workgroup computes a tile of BI x BJ sums, D[i][j] = sum_k A[i][k] B[j][k], 64 of
// k at a time. The tiles of A and B go from global memory straight into LDS (buffer
// loads with the LDS as their target, 16 bytes a lane), into one of two or three stages while the
// matrix instructions work on another. Two layouts of an operand in memory:
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

// Loads of a tile of R rows and 64 k of a K-contiguous operand (one tensor, or two, each half of
// the tile's rows) into a stage, step after step. NW waves.
template <int R, int NW, int kParts>
struct LoadRows {
  static constexpr int kLoads = R / 8 / NW;  // of a wave: 8 rows each
  __amdgpu_buffer_rsrc_t part[kParts];       // from the tile's first row on
  uint32_t k, K, step, off;  // the lane's next k; bytes between a wave's loads; the lane's offset

  // row0 < rows: the tile's first row; 256 rows are less than 2^31 bytes apart
  __device__ __forceinline__ void start(const void* const (&src)[kParts], int64_t ld, int64_t rows,
                                        int64_t row0, int64_t K_, int64_t k0, int wave, int lane) {
    const int r = 8 * wave + (lane >> 3);
    K = (uint32_t)K_;
    k = (uint32_t)k0 + ((lane & 7) ^ ((r >> 1) & 7)) * 8;
    off = (uint32_t)(r * ld + k) * 2;
    step = (uint32_t)(8 * NW * ld * 2);
    const int64_t left = ((rows - row0 - 1) * ld + K_) * 2;
    const uint32_t range = left < (int64_t)kOutOfRange ? (uint32_t)left : kOutOfRange;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
      part[i] = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>((const uint8_t*)src[i] + row0 * ld * 2), 0, (int)range, 0x00020000);
  }
  __device__ __forceinline__ void load(uint8_t* stage, int wave) {
    const uint32_t o = k < K ? off : kOutOfRange;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int h = i * kParts / kLoads;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          part[h], (lds_byte*)(stage + (wave + NW * i) * 1024), 16,
          o + (uint32_t)(i - h * kLoads / kParts) * step, 0, 0, 0);
    }
    k += kStepK;
    off += kStepK * 2;
  }
};

// Loads of a tile of 64 k and R columns of a K-major operand (one tensor, or two, one after the
// other along k, the first padded to a multiple of 64 k) into a stage, step after step.
template <int R, int NW, int kParts>
struct LoadColumns {
  static constexpr int kRowsPer = 512 / R;               // k of a load
  static constexpr int kLoads = kStepK / kRowsPer / NW;  // of a wave
  const uint8_t* p;  // the first tensor's row 0, at the tile's columns
  int64_t second;
  int ld2, k, K, Kp, end, width;
  uint32_t step, off;

  // K: the rows of a tensor, Kp: of the first and its padding, k1: where this sum ends (a step beyond
  // it loads zeros); 64 rows are less than 2^31 bytes apart
  __device__ __forceinline__ void start(const void* const (&src)[kParts], int64_t ld, int64_t cols,
                                        int64_t col0, int64_t K_, int64_t Kp_, int64_t k0,
                                        int64_t k1, int wave, int lane) {
    const int r = wave * kRowsPer + lane / (R / 8);
    const int f = (r & 3) | ((r >> 3) & 1) << 2;
    ld2 = (int)(ld * 2);
    k = (int)k0;
    K = (int)K_;
    Kp = (int)Kp_;
    end = (int)k1;
    width = (int)(cols - col0) * 2;
    off = (uint32_t)(r * ld2) + (uint32_t)(((lane % (R / 8)) ^ (f << 1)) * 16);
    step = (uint32_t)(NW * kRowsPer * ld2);
    p = (const uint8_t*)src[0] + col0 * 2;
    // the second tensor's distance, less the first one's padded rows: row k - Kp of it is row k of
    // the first, this much further on
    second = kParts == 2 ? (int64_t)(uintptr_t)src[kParts - 1] - (int64_t)(uintptr_t)src[0] - Kp_ * ld * 2 : 0;
  }
  __device__ __forceinline__ void load(uint8_t* stage, int wave) {
    const bool more = kParts == 2 && k >= Kp;
    int left = K - k + (more ? Kp : 0);
    left = left < end - k ? left : end - k;
    left = left < kStepK ? left : kStepK;
    const int range = (left - 1) * ld2 + width;
    const auto r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(p + (int64_t)k * ld2 + (more ? second : 0)), 0, left > 0 ? range : 0,
        0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_byte*)(stage + (wave + NW * i) * 1024), 16,
                                               off + (uint32_t)i * step, 0, 0, 0);
    k += kStepK;
  }
};

// Fragments of a stage: N of 16 rows each, k step ks (32 k). kHalf: the second half of the
// fragments is that many rows further on (the rows of the second tensor), 0: they follow on.
template <class T, int N, int kHalf>
struct ReadRows {
  static constexpr int kReads = N;  // LDS reads of a k step
  uint32_t at;
  __device__ __forceinline__ void start(int row0, int lane) {
    const int r = lane & 15, q = lane >> 4;
    at = (uint32_t)((row0 + r) * 128 + ((q ^ (r >> 1)) << 4));
  }
  __device__ __forceinline__ typename T::vec8 get(const uint8_t* stage, int i, int ks) const {
    const int row = kHalf == 0 || i < N / 2 ? 16 * i : kHalf + 16 * (i - N / 2);
    return *(const typename T::vec8*)(stage + (at ^ (uint32_t)(ks * 64)) + row * 128);
  }
};
template <class T, int N, int R>
struct ReadColumns {
  static constexpr int kReads = 2 * N;
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

// Waits until at most kPending of a wave's loads into LDS are under way and its LDS reads are
// done, then for the other waves.
template <int kPending>
__device__ __forceinline__ void stage_ready() {
  static_assert(kPending < 64);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kPending) : "memory");
}

// Before a wave ends, and with its workgroup LDS becomes another's.
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The order of a quarter step's instructions: LDS reads behind the first of the matrix instructions, so
// that they are done when the quarter is, loads spread over all of them.
template <int kMfma, int kReads, int kLoads>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < kMfma; ++i) {
#pragma unroll
    for (int n = kReads * i / kMfma; n < kReads * (i + 1) / kMfma; ++n)
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
    for (int n = kLoads * i / kMfma; n < kLoads * (i + 1) / kMfma; ++n)
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  }
}

// The sums of a wave's tile over `steps` steps of 64 k: acc[i][j] += A fragment i times B fragment j.
// load(s) issues a wave's kLoads loads of the next step's tiles into stage s (beyond the last step: of
// zeros, so that the number under way is always the same). There are S stages.
//
// A half step (32 k) multiplies the lower half of A's fragments, then the upper half; each quarter
// reads what the next one needs (the upper half; or the next half step's B and lower half), so that
// half of A's fragments and two sets of B's are held, not two of both: the registers just last, and one
// spilled to memory would cost more than any wait. A step's tiles are loaded S steps ahead: the one wait
// and barrier of a step stands before its last quarter, after which the stage that all waves
// have read takes the tiles S steps on.
template <class T, int NI, int NJ, int kLoads, int S, class ReadA, class ReadB, class Load>
__device__ __forceinline__ void sum_tiles(f32x4 (&acc)[NI][NJ], uint8_t* const (&sa)[S],
                                          uint8_t* const (&sb)[S], const ReadA& ra, const ReadB& rb,
                                          Load load, int steps) {
  typedef typename T::vec8 Vec;
  constexpr int H = NI / 2, kReadsA = ReadA::kReads / 2, kReadsB = ReadB::kReads;
  Vec lo[H], hi[H], b[2][NJ];
  const auto read_first = [&](int s, int ks) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) b[ks][j] = rb.get(sb[s], j, ks);
#pragma unroll
    for (int i = 0; i < H; ++i) lo[i] = ra.get(sa[s], i, ks);
  };
  const auto read_upper = [&](int s, int ks) {
#pragma unroll
    for (int i = 0; i < H; ++i) hi[i] = ra.get(sa[s], H + i, ks);
  };
  const auto multiply = [&](const Vec(&a)[H], int first, int ks) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[first + i][j] = T::mfma(a[i], b[ks][j], acc[first + i][j]);
  };
#pragma unroll
  for (int i = 0; i < S; ++i) load(i);
  stage_ready<(S - 1) * kLoads>();
  read_first(0, 0);
  // whole rounds of the stages (steps beyond the last are of zeros), so that the loop has one exit and
  // the sums stay in their registers
  for (int n = 0; n < steps; n += S) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      read_upper(s, 0);
      multiply(lo, 0, 0);
      interleave<H * NJ, kReadsA, 0>();
      read_first(s, 1);
      multiply(hi, H, 0);
      interleave<H * NJ, kReadsA + kReadsB, 0>();
      read_upper(s, 1);
      multiply(lo, 0, 1);
      interleave<H * NJ, kReadsA, 0>();
      stage_ready<(S - 2) * kLoads>();
      load(s);
      read_first((s + 1) % S, 0);
      multiply(hi, H, 1);
      interleave<H * NJ, kReadsA + kReadsB, kLoads>();
    }
  }
  loads_done();
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
