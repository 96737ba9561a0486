// Launchers of the block pack / unpack kernels, the gated feed-forward block,
// the products with 4-bit weights, and what stands around the block in a training
// step (block.hip, gated.hip, weights4.hip, norm.hip, linear.hip, adamw.hip), and
// the element types and narrow formats that they share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hobflops.h"

namespace hobflops {

// index of a narrow format in the kernels' template arguments
enum { kE4M3 = 0, kE5M2 = 1, kE2M1 = 2 };

// src / dst: [rows][cols] values of a type, rows ld values apart; codes dense,
// scales [rows][ceil(cols / group)] (group 32 and powers of two for 8-bit codes)
struct BlockTensor {
  const void* values;
  int type;
  int64_t rows, cols, ld;
  uint8_t* codes;
  void* scales;
  int group, scale;
};
hipError_t launch_block_pack(const BlockTensor& t, int fmt, hipStream_t stream);
hipError_t launch_block_unpack(const BlockTensor& t, int fmt, hipStream_t stream);

struct GatedBlocks {  // 8-bit codes [T][F] or [T][D] and their scale bytes
  uint8_t* codes;
  uint8_t* scales;
};
struct GatedForward {
  const void *x, *w_gate, *w_up;
  void* h;
  GatedBlocks gate, up;  // null codes: none are kept
  void* workspace;
};
struct GatedBackward {
  const void *dh, *w_gate, *w_up;
  GatedBlocks x, gate, up;
  void *dx, *dw_gate, *dw_up;
  void* workspace;
};
int64_t gated_forward_workspace(const hobflops_gated_desc& d);
int64_t gated_backward_workspace(const hobflops_gated_desc& d);
// fmt: kE4M3, kE5M2 or -1
hipError_t launch_gated_forward(const hobflops_gated_desc& d, const GatedForward& p, int fmt,
                                hipStream_t stream);
hipError_t launch_gated_backward(const hobflops_gated_desc& d, const GatedBackward& p, int fmt,
                                 hipStream_t stream);

struct W4Matrix {
  const uint8_t* codes;  // [N][ceil(K / 2)]
  const void* scales;    // [N][ceil(K / group)]
};
struct W4Product {
  const void* x;
  int type;
  int64_t T, K, N, ldx, ldy;
  W4Matrix w, w_up;  // w_up.codes null: one projection
  int group, scale, act;
  void* y;
};
hipError_t launch_w4(const W4Product& p, hipStream_t stream);

struct LayerNorm {  // a forward or a backward call; dx rows are dense
  int64_t rows, cols, ldx, ldy, ld_add;
  int type, wtype;
  double eps;
  const void *x, *w, *b, *dy, *add;
  void *y, *dx, *dw, *db;
  float *mean, *rstd;
  void* workspace;
};
int64_t norm_backward_workspace(int64_t rows, int64_t cols, int type);
hipError_t launch_norm_forward(const LayerNorm& p, hipStream_t stream);
hipError_t launch_norm_backward(const LayerNorm& p, hipStream_t stream);

struct LinearForward {
  const void *x, *w, *bias, *residual;
  void *y, *z, *workspace;
};
struct LinearBackward {
  const void *dy, *x, *w, *z;
  void *dx, *dw, *db, *workspace;  // null: not asked for
};
struct LinearNeed {
  bool dx, dw, db;
};
int64_t linear_forward_workspace(const hobflops_linear_desc& d);
int64_t linear_backward_workspace(const hobflops_linear_desc& d, const LinearNeed& need);
hipError_t launch_linear_forward(const hobflops_linear_desc& d, const LinearForward& p, hipStream_t stream);
hipError_t launch_linear_backward(const hobflops_linear_desc& d, const LinearBackward& p, hipStream_t stream);

struct AdamwState {  // scales null: float32
  void *m, *v;
  uint8_t *m_scales, *v_scales;
};
// fmt: kE4M3, kE5M2 or -1
hipError_t launch_adamw(const hobflops_adamw_desc& d, const hobflops_adamw_tensor* tensors, int count, int fmt,
                        const AdamwState& state, hipStream_t stream);

}  // namespace hobflops
