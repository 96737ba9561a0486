"""Products with 4-bit weights where x and the scales are far from 1 and their products are not: no sum
leaves float32's range that the formula's own terms do not leave.

Tolerance, derived: that of test_gpu_w4, and for products and sums below 2^-126 float32's smallest step,
2^-149, for each of K terms: once as a term and once in a sum, under what is left of a scale, below 2."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say
from test_gpu_w4 import ACT, EPS, TINY, TYPES, UNIT

pytestmark = pytest.mark.gpu
# a call of each kernel: T, N, K
CALLS = [(1, 40, 256), (5, 260, 520), (16, 33, 11264), (20, 8200, 264), (1, 9, 37)]


def _case(hf, T, N, K, dtype, group, scale, ex, es, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.rand((T, K), generator=g) + 1) * torch.where(torch.rand((T, K), generator=g) < 0.5, -1.0, 1.0)
    x = (x * 2.0 ** ex).to(TYPES[dtype])
    packed = torch.randint(0, 256, (N, (K + 1) // 2), generator=g, dtype=torch.uint8)
    groups = -(-K // group)
    if scale == "pow2":
        s = torch.randint(es + 125, es + 128, (N, groups), generator=g).to(torch.uint8)
        f = np.exp2(s.double().numpy() - 127)
    else:
        s = ((torch.rand((N, groups), generator=g) + 1).double() * 2.0 ** es).to(
            torch.bfloat16 if scale == "bf16" else torch.float32)
        f = s.double().numpy()
    w = ref.unpack(ref.nibbles(packed.numpy(), K), f, (2, 1), group)
    return x, packed.cuda(), s.cuda(), torch.from_numpy(w)


@pytest.mark.parametrize("T,N,K", CALLS)
@pytest.mark.parametrize("group,scale", [(32, "pow2"), (32, "f32"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("dtype,ex,es", [("bf16", 126, -100), ("bf16", 126, -125), ("bf16", -120, 100),
                                         ("bf16", -126, 110), ("bf16", 100, -110), ("f16", 14, -30),
                                         ("f16", -14, 10), ("f16", -24, 20)])
def test_far_from_one(T, N, K, group, scale, dtype, ex, es):
    hf = need_gpu()
    say("w4 far from one", T, N, K, group, scale, dtype, ex, es)
    x, codes, s, w = _case(hf, T, N, K, dtype, group, scale, ex, es, 41)
    y = hf.w4_linear(x.cuda(), codes, s, group=group).double().cpu()
    want, size = x.double() @ w.T, x.double().abs() @ w.abs().T
    if dtype == "f16":    # what float16 holds of it
        far = size > 60000
        y, want, size = (torch.where(far, torch.zeros_like(t), t) for t in (y, want, size))
    bound = (K + 4) * EPS * size + UNIT[dtype] * want.abs() + TINY[dtype] + 4 * K * 2.0 ** -149
    assert ((y - want).abs() <= bound).all()


@pytest.mark.parametrize("T,N,K", CALLS)
@pytest.mark.parametrize("group,scale", [(32, "pow2"), (32, "f32"), (64, "bf16")])
def test_gated_far_from_one(T, N, K, group, scale):
    """The gate near 1, the other projection large: x of about 2^126."""
    hf = need_gpu()
    x, cg, sg, wg = _case(hf, T, N, K, "bf16", group, scale, 126, -125, 42)
    _, cu, su, wu = _case(hf, T, N, K, "bf16", group, scale, 126, -110, 43)
    h = hf.w4_gated(x.cuda(), cg, sg, cu, su, 0, group=group).double().cpu()
    x = x.double()
    g, u = x @ wg.T, x @ wu.T
    eg, eu = ((K + 4) * EPS * (x.abs() @ w.abs().T) for w in (wg, wu))
    a = g * torch.sigmoid(g)
    e = (1.13 * eg + ACT * g.abs()) * (u.abs() + eu) + a.abs() * eu
    assert ((h - a * u).abs() <= e + UNIT["bf16"] * (a * u).abs()).all()
