"""The linear layer's gradients where z, kept in 16 bits for the backward pass, is rounded to an infinity: the
activations' slopes are 0 and 1 there, as they are of every z of some hundred.

Tolerances as in the linear layer's own tests: a float32 sum of n products is n 2^-23 sum |a b| off, dz and the
results are rounded to their type, half a step each; slopes at these z are exact, of the others 2^-19 (1 + |z|) off.
"""
import pytest
import torch

import step_ref as ref
from gpu_util import need_gpu, say
from test_gpu_linear import ACT, EPS, TYPES, _act, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N", [(1, 64, 40), (5, 37, 31), (20, 8192, 64), (300, 520, 520), (2048, 512, 1400)])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_z_beyond_float16(T, K, N, act):
    """Tokens and outputs whose z is some -7e4 or 7e4: y is finite on the negative side, gradients everywhere."""
    hf = need_gpu()
    say("linear far", T, K, N, act)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(T, K, generator=g)
    w = torch.randn(N, K, generator=g) * K ** -0.5
    x[T - 1, 0], x[0, 1 % K] = 300.0, 280.0
    w[N - 1, 0], w[1, 0], w[0, 1 % K], w[2, 1 % K] = -235.0, 240.0, -250.0, 245.0
    if T == 1:
        x[0, 1 % K] = 0.0
    x, w = x.half().cuda(), w.half().cuda()
    dy = (torch.randn(T, N, generator=g) / 4).half().cuda()
    y, kept = hf.linear(x, w, None, act, save=True)
    z = x.double() @ w.double().T
    far = z.abs() > 65600
    assert (far & (z < 0)).any() and (far & (z > 0)).any() and kept[far].isinf().all() and kept[~far].isfinite().all()
    assert (y[far & (z < 0)] == 0).all()
    dx, dw, db = hf.linear_backward(dy, x, w, kept, act)
    near = torch.where(far, torch.zeros_like(z), kept.double())
    slope = torch.where(far, (z > 0).double(), _act(near, act)[1])
    dz, x, w, dy = dy.double() * slope, x.double(), w.double(), dy.double().abs()
    err = torch.where(far, torch.zeros_like(z), ACT * (1 + near.abs()) * dy)
    half = ref.HALF["f16"] * dz.abs() + ref.TINY["f16"] + err
    mag = dz.abs() + half
    _check(dx, dz @ w, half @ w.abs() + N * EPS * (mag @ w.abs()), "f16", "dx")
    _check(dw, dz.T @ x, half.T @ x.abs() + T * EPS * (mag.T @ x.abs()), "f16", "dw")
    _check(db, dz.sum(0), err.sum(0) + T * EPS * dz.abs().sum(0), "f16", "db")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_infinite_z(dtype, act):
    """The slopes of an infinite z are those of a far one, bit for bit; of NaN they are NaN."""
    hf = need_gpu()
    g = torch.Generator().manual_seed(2)
    x, w, dy, z = (torch.randn(*s, generator=g).to(TYPES[dtype]).cuda() for s in ((9, 72), (41, 72), (9, 41), (9, 41)))
    far, inf = z.clone(), z.clone()
    for at, sign in (((0, 0), 1), ((3, 17), -1), ((8, 40), -1), ((8, 39), 1)):
        far[at], inf[at] = sign * 1e4, sign * float("inf")
    want = hf.linear_backward(dy, x, w, far, act)
    assert all(t.isfinite().all() for t in want)
    assert all(torch.equal(a, b) for a, b in zip(hf.linear_backward(dy, x, w, inf, act), want))
    inf[4, 20] = float("nan")
    dx, dw, db = hf.linear_backward(dy, x, w, inf, act)
    assert dx[4].isnan().all() and dw[20].isnan().all() and db[20].isnan()
    keep = torch.arange(9, device="cuda") != 4
    assert torch.equal(dx[keep], want[0][keep])
