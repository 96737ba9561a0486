"""The kernels that a call of the linear layer runs, by its plan (host code of the library, compiled on its own)."""
import os
import subprocess

from paper_2007_06563_amd import build

SRC = r"""
#include <stdio.h>
#include "linear_plan.hpp"
using namespace hobflops;
int main() {
  hobflops_linear_desc d{};
  long long v[7];
  while (scanf("%lld %lld %lld %lld %lld %lld %lld %d %d", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6, &d.act, &d.align) == 9) {
    d.T = v[0]; d.K = v[1]; d.N = v[2]; d.ldx = v[3]; d.ldw = v[4]; d.ldy = v[5]; d.ldr = v[6];
    d.type = HOBFLOPS_TYPE_BF16;
    const ForwardPlan f = plan_forward(d);
    int64_t per = 0;
    if (f.direct >= 0) {
      printf("direct%d\n", f.direct);
    } else {
      const int tail = f.x >= 0 && f.w >= 0 ? 0 : (int)(d.K % 8);
      const int64_t K = f.x >= 0 && f.w >= 0 ? round_up(d.K, 8) : d.K - tail;
      printf("forward%d%s%s%s%s\n", f.tiles.kind, splits_of(K > 0 ? K : 1, f.tiles.splits, &per) > 1 ? " parts" : "",
             tail ? " tail" : "", f.x >= 0 ? " x" : "", f.w >= 0 ? " w" : "");
    }
    const BackwardPlan b = plan_backward(d, LinearNeed{true, true, true});
    printf("dx%d%s dw%d%s%s%s%s%s\n", b.dx.kind, splits_of(b.Np, b.dx.splits, &per) > 1 ? " parts" : "", b.dw.kind,
           splits_of(d.T, b.dw.splits, &per) > 1 ? " parts" : "", b.dx.kind == b.dw.kind ? " joint" : " apart",
           b.dz >= 0 ? " dz" : "", b.x >= 0 ? " x" : "", b.w >= 0 ? " w" : "");
  }
}
"""


def align(offset):
    """The alignment in bytes of tensors that begin `offset` 16-bit values past 16 bytes."""
    return (offset * 2 | 16) & -(offset * 2 | 16)


def plans(calls, folder):
    """(forward, backward) of calls (T, K, N, (ldx, ldw, ldy, ldr) or None, offset, act or None), as the plan says."""
    src, exe = os.path.join(folder, "plan.hip"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(SRC)
    r = subprocess.run([build.HIPCC, "-std=c++17", "--cuda-host-only", "-I", os.path.join(build.HERE, "csrc"), "-I",
                        os.path.join(build.ROOT, "include"), src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = []
    for T, K, N, lds, off, act in calls:
        ldx, ldw, ldy, ldr = lds or (K, K, N, N)
        lines.append(" ".join(map(str, (T, K, N, ldx, ldw, ldy, ldr, -1 if act is None else act, align(off)))))
    r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True)
    out = r.stdout.splitlines()
    assert r.returncode == 0 and len(out) == 2 * len(calls)
    return list(zip(out[::2], out[1::2]))


# T, K, N, (ldx, ldw, ldy, ldr) or those of dense rows, offset in elements, activation
def _lds(N, ldx, ldw):
    return ldx, ldw, N, N


SHAPES = [
    # straight from memory, by tile
    (1, 64, 64, None, 0, 0), (195, 64, 320, None, 2, None), (631, 64, 392, _lds(392, 72, 64), 1, None),
    (134, 64, 832, _lds(832, 72, 64), 1, None), (356, 64, 704, None, 1, None), (483, 69, 1034, _lds(1034, 77, 69), 0, 0),
    # 256 x 256: whole, in parts, the last K % 8 apart, one operand copied and one not, both
    (516, 72, 13528, None, 0, 0), (2582, 4296, 1560, None, 0, None), (647, 66, 10964, None, 0, None), (1543, 4526, 2614, None, 0, 0),
    (2875, 70, 2982, _lds(2982, 78, 71), 0, None), (2566, 69, 3076, _lds(3076, 69, 70), 0, 0), (515, 79, 13715, None, 0, None),
    (1986, 6839, 2149, None, 0, None),
    # 128 x 128, two on a CU
    (135, 64, 8320, None, 2, None), (1361, 5712, 920, None, 2, 0), (129, 92, 8881, None, 0, 0), (1345, 5962, 1027, None, 0, None),
    (276, 68, 5736, _lds(5736, 76, 69), 0, 0), (258, 66, 5696, _lds(5696, 67, 66), 0, 0), (136, 65, 8394, _lds(8394, 67, 67), 0, None),
    # 128 x 128, four stages
    (548, 136, 3440, None, 2, 0), (794, 3408, 1296, None, 0, 0), (545, 134, 3302, None, 0, 0), (1156, 3390, 844, None, 0, 0),
    (265, 130, 6013, _lds(6013, 132, 131), 0, 0), (528, 139, 3762, _lds(3762, 141, 140), 0, 0), (1153, 159, 1606, None, 0, 0),
    # 64 x 128, six
    (162, 64, 704, None, 0, None), (326, 8320, 768, _lds(768, 8320, 8322), 0, 0), (193, 66, 1224, _lds(1224, 68, 74), 0, 0),
    (610, 7366, 408, None, 2, None), (1029, 68, 990, _lds(990, 70, 69), 0, 0), (1746, 70, 588, _lds(588, 71, 78), 0, 0),
    (135, 69, 5574, None, 0, None),
    # 64 x 64, eight
    (420, 320, 640, _lds(640, 320, 328), 2, 0), (17, 15576, 64, _lds(64, 15576, 15584), 0, None), (527, 310, 642, _lds(642, 318, 318), 0, None),
    (27, 14708, 64, None, 0, None), (19, 14198, 70, _lds(70, 14198, 14199), 0, None), (1330, 5438, 412, _lds(412, 5439, 5440), 0, 0),
    (653, 2240, 832, None, 1, 0),
    # the gradients' products: one kind and launch for both, in parts or not
    (267, 13656, 144, _lds(144, 13664, 13656), 0, None), (265, 13408, 134, _lds(134, 13408, 13409), 2, 0), (3415, 1576, 280, None, 0, None),
    (129, 2864, 1600, None, 0, None), (1124, 2368, 64, None, 0, None), (3, 136, 15184, None, 0, None),
    (1732, 192, 1856, _lds(1856, 192, 200), 0, None), (853, 64, 64, None, 0, None), (931, 72, 920, None, 0, None),
    # a launch each
    (6722, 1808, 1144, None, 0, None), (872, 1656, 8408, None, 0, None), (165, 1944, 5200, None, 0, None), (2724, 4408, 72, None, 0, None),
    (265, 7984, 768, None, 0, None), (7238, 832, 4928, _lds(4928, 840, 840), 0, None),
]
