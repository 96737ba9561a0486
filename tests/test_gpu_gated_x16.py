"""Checkpoints of x that stand for values beyond the type's largest: rounding to a block's code takes
float16 |x| of 63488 and more in (4, 3), 61440 and more in (5, 2), to 65536, and bfloat16 of 2^112 times
these to 2^128.

Tolerance, derived: that of test_gpu_gated, and for x, an operand in 16 bits, a relative UNIT: the type's
largest value taken for the power of two above it (all other values of such blocks are the type's)."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say
from test_gpu_gated import EPS, TINY, TYPES, UNIT, _blocks, _gradients, _make

pytestmark = pytest.mark.gpu
TOP = [65504.0, -65504.0, 63488.0, -61440.0, 63456.0, 61408.0, 57344.0]


def _case(hf, T, D, F, f, x, dtype="f16"):
    gt, wg = _make(F, D, dtype, 31, 2.0 ** -6)
    ut, wu = _make(F, D, dtype, 32, 2.0 ** -6)
    dt, dh = _make(T, F, dtype, 33, 2.0 ** -10)
    blocks = [hf.block_pack(t.cuda(), f) for t in (
        x, torch.randn(T, F, generator=torch.Generator().manual_seed(34)),
        torch.randn(T, F, generator=torch.Generator().manual_seed(35)))]
    saved = hf.GatedSaved(*blocks, hf.fmt(f))
    return (gt, ut, dt), saved, (dh, wg, wu, *(_blocks(hf, (b, f), 0)[0] for b in blocks))


@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("f", [(4, 3), (5, 2)])
@pytest.mark.parametrize("dtype,up", [("f16", 1.0), ("bf16", 2.0 ** 112)])
@pytest.mark.parametrize("T,D,F", [(5, 40, 33), (3, 37, 64), (300, 136, 264)])
def test_largest_x(T, D, F, dtype, up, f, act):
    hf = need_gpu()
    say("largest x", T, D, F, dtype, f, act)
    x = torch.randn(T, D, generator=torch.Generator().manual_seed(30))
    for i, v in enumerate(TOP):
        x[i % T, (11 * i) % D] = v if dtype == "f16" else np.clip(v, -65280, 65280)
    x = (x.double() * up).to(TYPES[dtype])
    assert x.isfinite().all()
    (gt, ut, dt), saved, (dh, wg, wu, xq, gq, uq) = _case(hf, T, D, F, f, x, dtype)
    assert np.abs(xq).max() == 65536.0 * up
    grads = hf.gated_backward(dt, saved, gt, ut, act)
    a, da = ref.act(gq, act)
    weights = (dh * uq * da, dh * a)
    for i, (got, (want, bound)) in enumerate(zip(grads, _gradients(dh, wg, wu, xq, gq, uq, dtype, act))):
        if i:  # x's own rounding, of sums in which each gradient is off by its rounding as well
            v = np.abs(weights[i - 1]) * (1 + UNIT[dtype]) + 2 * TINY[dtype]
            bound = bound + v.T @ (UNIT[dtype] * np.abs(xq)) * (1 + T * EPS)
        got = got.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("f", [(4, 3), (5, 2)])
def test_what_float16_cannot_hold(f):
    """Infinities keep their column of the weights' gradients alone, and so do block values above
    65536, which only x of another type has: infinity, as float16 rounds them."""
    hf = need_gpu()
    T, D, F = 5, 72, 33
    x = torch.randn(T, D, generator=torch.Generator().manual_seed(36))
    base = x.clone()
    x[2, 3], x[4, 40] = float("inf"), 1e6
    (gt, ut, dt), saved, _ = _case(hf, T, D, F, f, base)
    with_inf = hf.GatedSaved(hf.block_pack(x.cuda(), f), saved.gate, saved.up, saved.fmt)
    group = torch.arange(D) // 32 == 1     # 1e6 changes the scale of its group's other values
    clean = ~group
    clean[3] = False
    for a, b in zip(hf.gated_backward(dt, saved, gt, ut)[1:], hf.gated_backward(dt, with_inf, gt, ut)[1:]):
        a, b = a.cpu(), b.cpu()
        assert torch.equal(a[:, clean], b[:, clean])
        assert not b[:, [3, 40]].isfinite().any()
        group[40] = False
        assert b[:, group].isfinite().all()
