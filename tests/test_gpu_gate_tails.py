"""The activations far from zero, where they are small beside their argument, against 64 bits under
relative bounds: forward, gradients and the product with 4-bit weights.

Every product here has one term, a power of two times a value of the type, so the argument g is exact.
Tolerance, derived: the exponential's argument (g, or g^2 / 2 of at most 41) is rounded to float32
by at most 2^-23 of itself and the function follows with a relative 41 * 2^-23 < 2^-17; erfc, exp, the
reciprocal and the products are a few units of 2^-23 each, act' adds two terms whose sum is at
least a third of them: 2^-14 in all. A sigmoid below 2^-126 has a step of 2^-149. Outputs and, in the
gradients, one operand are rounded to the type: UNIT each, TINY where it has no smaller step (for an
operand in bfloat16 the smallest normal value, 2^-126)."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say
from test_gpu_gated import TINY, TYPES, UNIT, _blocks

pytestmark = pytest.mark.gpu
REL, STEP = 2.0 ** -14, 2.0 ** -149
LOW = {0: (-100.0, -2.0), 1: (-9.0, -2.0)}   # SiLU, GELU
# what the up projection multiplies by, to bring small values into the type
UP = {("bf16", 0): 2.0 ** 60, ("bf16", 1): 2.0 ** 12, ("f16", 0): 2.0 ** 14, ("f16", 1): 2.0 ** 14}


def _g(act, dtype, n=257):
    return torch.linspace(*LOW[act], n).to(TYPES[dtype])


def _check(got, want, dtype, u, roundings=1):
    got = got.double().cpu().numpy().ravel()
    bound = (REL + roundings * UNIT[dtype]) * (1 + UNIT[dtype]) * np.abs(want) + np.abs(u) * STEP
    tiny = 2.0 ** -126 if dtype == "bf16" and roundings > 1 else roundings * TINY[dtype]
    assert (np.abs(got - want) <= bound + tiny).all(), float((np.abs(got - want) / (bound + tiny + 1e-300)).max())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", [0, 1])
def test_forward(act, dtype):
    hf = need_gpu()
    say("tails forward", act, dtype)
    g, s = _g(act, dtype), UP[dtype, act]
    x = torch.zeros(1, 8, dtype=g.dtype)
    x[0, 0] = 1.0
    wg = torch.zeros(len(g), 8, dtype=g.dtype)
    wu = wg.clone()
    wg[:, 0], wu[:, 0] = g, s
    h = hf.gated_forward(x.cuda(), wg.cuda(), wu.cuda(), act)
    g = g.double().numpy()
    _check(h, ref.act(g, act)[0] * s, dtype, g * s)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", [0, 1])
def test_gradients(act, dtype):
    """One token with x = 1: the weights' gradients are dg and du."""
    hf = need_gpu()
    say("tails gradients", act, dtype)
    f, s = (4, 3), 2.0 ** 10
    g = _g(act, dtype).reshape(1, -1)
    g = g[:, :g.shape[1] // 32 * 32].cuda()
    gate = hf.block_pack(g, f)
    gq = _blocks(hf, (gate, f), 0)[0].ravel()
    u = torch.full_like(g, 1.5)
    x = torch.zeros(1, 8, dtype=g.dtype, device="cuda")
    x[0, 0] = 1.0
    dh = torch.full_like(g, s)
    w = torch.zeros(g.shape[1], 8, dtype=g.dtype, device="cuda")
    saved = hf.GatedSaved(hf.block_pack(x, f), gate, hf.block_pack(u, f), hf.fmt(f))
    _, dwg, dwu = hf.gated_backward(dh, saved, w, w, act)
    a, da = ref.act(gq, act)
    _check(dwg[:, 0], s * 1.5 * da, dtype, 1.5 * s * (1 + np.abs(gq)), 2)
    _check(dwu[:, 0], s * a, dtype, s * gq, 2)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("T,N", [(1, 16), (16, 40), (20, 8200)])
def test_w4_gated(T, N, act, dtype):
    hf = need_gpu()
    say("tails w4", T, N, act, dtype)
    g, s = _g(act, dtype, T), UP[dtype, act]
    x = torch.zeros(T, 64, dtype=g.dtype)
    x[:, 0], x[:, 33] = g, 1.0
    codes = torch.zeros(N, 32, dtype=torch.uint8)
    cg, cu = codes.clone(), codes.clone()
    cg[:, 0] = 2                             # 1.0 at k = 0
    cu[:, 16] = 2 << 4                       # and at k = 33
    sg = torch.ones(N, 2)
    su = torch.ones(N, 2) * s
    h = hf.w4_gated(x.cuda(), cg.cuda(), sg.cuda(), cu.cuda(), su.cuda(), act)
    assert (h == h[:, :1]).all()
    g = g.double().numpy()
    _check(h[:, 0], ref.act(g, act)[0] * s, dtype, g * s)
