// Which kernel a call of the linear layer runs, and what its workspace holds: host code alone, so that the choice can be looked
// at without a GPU.
#pragma once
#include <stdint.h>

#include "block.hpp"
#include "gemm.hpp"
#include "tiles.hpp"

namespace hobflops {

constexpr int kNoAct = HOBFLOPS_GATE_NONE;

// Reading rows that do not begin on lines of 128 bytes takes a third more, rows at odd values twice as long (direct_kernel, 333 x
// 8192 -> 1000: 21 us, of 8200 values 26, of 8193 37; in tiles 512 x 4104 -> 4096 32, of 4096 values 23).
inline double row_factor(int64_t ld, int align) { return ld % 2 != 0 || align == 2 ? 2.0 : ld % 64 != 0 ? 1.33 : 1.0; }
// The tiles of a product through LDS and the parts of its sum, by an estimate of their time in microseconds: rounds of
// workgroups, each its steps of 64 k and some more to start and end; the parts of a sum are written and read
// once more in float32, 4 TB/s, and joined in a launch, eight at a time. The kinds' times are those of the sizes that each is for, measured: of
// 4096 x 4096 -> 4096 (98 us), 2048 x 4096 -> 4096 (60, the others 84, 65 and 88), 1024 x 4096 -> 4096 (34; 78, 44, 46),
// 512 x 4096 -> 4096 (24; 76, 41, 28, 31) and 256 x 4096 -> 4096 (16). Steps of rows off the lines of memory take longer, as above.
struct Kind {
  int rows, cols, per_cu;
  double step, lead;
};
constexpr Kind kKinds[] = {{256, 256, 1, 1.42, 5}, {128, 128, 2, 0.8, 5}, {128, 128, 1, 0.45, 11}, {64, 128, 1, 0.31, 14}, {64, 64, 1, 0.17, 30}};
constexpr int kForwardKinds = 5, kGradKinds = 3;
struct Tiling {
  int kind, splits;
  int64_t groups;           // workgroups
  double each, join, us;    // the time of a workgroup, of the parts, of all
};
constexpr int kMostSplits = 128;
// The best of kinds first, .. last - 1. off: whether rows begin off the lines of memory.
inline Tiling plan_tiles(int64_t rows, int64_t cols, int64_t K, int first, int last, bool off = false) {
  const int64_t steps = (K + kStepK - 1) / kStepK;
  Tiling best{first, 1, 0, 0.0, 0.0, -1.0};
  for (int k = first; k < last; ++k) {
    const Kind& kind = kKinds[k];
    const int64_t slots = kind.per_cu * kCUs;
    const int64_t tiles = ((rows + kind.rows - 1) / kind.rows) * ((cols + kind.cols - 1) / kind.cols);
    for (int n = 1; n <= kMostSplits && (n == 1 || steps / n >= 3); n += 1 + n / 16) {
      const double rounds = (double)((tiles * n + slots - 1) / slots);
      const double each = ((double)((steps + n - 1) / n) * (off ? (k == 0 ? 1.17 : 1.33) : 1.0) + kind.lead) * kind.step;
      const double join = n > 1 ? 4.0 + 0.1 * n + (double)(2 * n) * rows * cols * 4.0 / 4e6 : 0.0;
      const double us = rounds * each + join;
      if (best.us < 0.0 || us < best.us) best = Tiling{k, n, tiles * n, each, join, us};
    }
  }
  return best;
}
// Of one launch with a's workgroups and then b's, of one kind: b's begin where a's leave CUs idle.
inline double pair_us(const Tiling& a, const Tiling& b) {
  const int64_t slots = kKinds[a.kind].per_cu * kCUs, rounds = (a.groups + slots - 1) / slots;
  const int64_t beside = (rounds * slots - a.groups) * (a.each > b.each ? (int64_t)(a.each / b.each) : 1);
  const int64_t left = b.groups > beside ? b.groups - beside : 0;
  const double t = (double)rounds * a.each + (double)((left + slots - 1) / slots) * b.each;
  const double alone = (double)(rounds - 1) * a.each + b.each;
  return (t > alone ? t : alone) + a.join + b.join;
}
// The tile of direct_kernel in 16 rows of W and 16 tokens, by an estimate: rounds of workgroups, one on each CU, which
// read their rows at 100 bytes a nanosecond, and start and end, the longer the larger the tile; or the weights from HBM, at
// the rate that the CUs in use leave of it (32 x 4096 -> 11264: 352 workgroups, 24 us; in tiles of 64 x 64 19). Measured, us, in the order
// of kDirect, and in tiles through LDS: 16 x 4096 -> 4096 8.5, 9.3, 10.7, 9.6, 12.0, 18.1, LDS 15.3; 64 x 4096 -> 4096
// 19.0, 15.5, 12.1, 10.7, 13.5, 18.4, LDS 17.3; 333 x 2730 -> 1000 24.5, 20.6, 19.2, 16.8, 13.0, 18.6, LDS 24.2;
// 1024 x 1024 -> 1024 33, 29, 19, 16, 13, 9.4, LDS 14.0; 2048 x 512 -> 1408 77, 66, 25, 38, 22, 18, LDS 10.0.
struct Direct {
  int ni, nj;
};
constexpr Direct kDirect[] = {{1, 1}, {1, 2}, {1, 4}, {2, 2}, {2, 4}, {4, 4}};
inline int plan_direct(int64_t N, int64_t T, int64_t K, double factor, double* us) {
  int best = 0;
  *us = -1.0;
  for (int i = 0; i < 6; ++i) {
    const Direct d = kDirect[i];
    if (d.nj > 1 && T <= 8 * d.nj) continue;  // more than half of the tokens would be nobody's
    const int64_t groups = ((N + 16 * d.ni - 1) / (16 * d.ni)) * ((T + 16 * d.nj - 1) / (16 * d.nj));
    const double rounds = (double)((groups + kCUs - 1) / kCUs);
    double t = rounds * (factor * (16 * (d.ni + d.nj)) * K * 2.0 / 100e3 + 1.0 + 0.18 * d.ni * d.nj);
    // the weights from HBM, 4.9 TB/s of full rounds; what is shorter of the two is not all hidden
    const double read = (double)N * K * 2.0 / 4.9e6 * rounds * kCUs / groups;
    t = t > read ? t + 0.1 * read : read + 0.1 * t;
    t += 3.0;
    if (*us < 0.0 || t < *us) {
      *us = t;
      best = i;
    }
  }
  return best;
}
// Rows that the products read in place.
inline bool in_place(int64_t cols, int64_t ld, int align) {
  return align >= 16 && cols % 8 == 0 && ld % 8 == 0 && ld < (int64_t)1 << 21;
}
inline int64_t splits_of(int64_t K, int splits, int64_t* per) {
  *per = round_up((K + splits - 1) / splits, kStepK);
  return (K + *per - 1) / *per;
}

struct ForwardPlan {
  int64_t x = -1, w = -1, part = -1, bytes = 0;
  Tiling tiles{0, 1};
  int direct = -1;  // of kDirect
};
// Rows that the forward product reads in place: loads of 16 bytes into LDS need addresses of whole words.
inline bool words(int64_t ld, int align) { return align >= 4 && ld % 2 == 0 && ld < (int64_t)1 << 21; }
// Values between the rows of a copy, whose last ones are zeros: rows that are not short begin on lines of memory.
inline int64_t copied_ld(int64_t K) { return round_up(K, K < 512 ? 8 : 64); }
inline ForwardPlan plan_forward(const hobflops_linear_desc& d) {
  ForwardPlan p;
  const double fx = row_factor(d.ldx, d.align), fw = row_factor(d.ldw, d.align);
  double direct = 0.0;
  const int i = plan_direct(d.N, d.T, d.K, fx > fw ? fx : fw, &direct);
  const bool x = words(d.ldx, d.align), w = words(d.ldw, d.align);  // in place
  p.tiles = plan_tiles(d.N, d.T, d.K, 0, kForwardKinds, (x && fx > 1.0) || (w && fw > 1.0));
  const double read = (double)d.N * d.K * 2.0 / 4.4e6 + 3.0;  // the weights from HBM
  double us = (p.tiles.us > read ? p.tiles.us : read) + (p.tiles.splits > 1 ? 4.0 : 0.0);  // (the second launch's start)
  // (rows that are not in place are copied in a launch of their own first)
  if (!x || !w) us += 4.0 + (double)(d.T + d.N) * d.K * 4.0 / 4e6;
  // (a tile through LDS would be three quarters nobody's tokens, and direct_kernel reads the weights at HBM's rate)
  if (direct < us || d.T <= 16) {
    p.direct = i;
    return p;
  }
  if (!x) p.x = take(&p.bytes, d.T * copied_ld(d.K) * 2);
  if (!w) p.w = take(&p.bytes, d.N * copied_ld(d.K) * 2);
  if (p.tiles.splits > 1) p.part = take(&p.bytes, p.tiles.splits * d.T * round_up(d.N, 4) * 4);
  return p;
}

struct BackwardPlan {
  int64_t x = -1, w = -1, dz = -1, db = -1, part_x = -1, part_w = -1, bytes = 0;
  int64_t Kp, Np;
  uint32_t parts = 1;  // of db
  Tiling dx{0, 1}, dw{0, 1};
};
// need: the gradients asked for
inline BackwardPlan plan_backward(const hobflops_linear_desc& d, const LinearNeed& need) {
  BackwardPlan p;
  p.Kp = round_up(d.K, 8);
  p.Np = round_up(d.N, 8);
  if (d.T == 0) return p;
  const bool products = need.dx || need.dw;
  if (products && (d.act != kNoAct || !in_place(d.N, d.ldy, d.align))) p.dz = take(&p.bytes, d.T * p.Np * 2);
  if (need.dw && !in_place(d.K, d.ldx, d.align)) p.x = take(&p.bytes, d.T * p.Kp * 2);
  if (need.dx && !in_place(d.K, d.ldw, d.align)) p.w = take(&p.bytes, d.N * p.Kp * 2);
  if (need.dx) p.dx = plan_tiles(d.T, d.K, p.Np, 0, kGradKinds);
  if (need.dw) p.dw = plan_tiles(d.N, d.K, d.T, 0, kGradKinds);
  if (need.dx && need.dw) {
    // the kinds that are best alone, a launch each, or one kind and launch for both (77 x 1022 -> 2731: 3 us less)
    double us = p.dx.us + p.dw.us + 3.0;
    if (p.dx.kind == p.dw.kind) us = pair_us(p.dx, p.dw);
    for (int k = 0; k < kGradKinds; ++k) {
      const Tiling a = plan_tiles(d.T, d.K, p.Np, k, k + 1), b = plan_tiles(d.N, d.K, d.T, k, k + 1);
      const double t = pair_us(a, b);
      if (t >= us) continue;
      us = t;
      p.dx = a;
      p.dw = b;
    }
  }
  if (need.dx && p.dx.splits > 1) p.part_x = take(&p.bytes, p.dx.splits * d.T * round_up(d.K, 4) * 4);
  if (need.dw && p.dw.splits > 1) p.part_w = take(&p.bytes, p.dw.splits * d.N * round_up(d.K, 4) * 4);
  const int64_t strips = (d.N + 255) / 256, most = (d.T + 7) / 8, wanted = (2048 + strips - 1) / strips;
  p.parts = (uint32_t)(most < wanted ? most : wanted);
  if (need.db) p.db = take(&p.bytes, (int64_t)p.parts * p.Np * 4);
  return p;
}

}  // namespace hobflops
