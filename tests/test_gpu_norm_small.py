"""Layer norm of rows whose squares are below float32's range (eps 0, or as small), against a plain 64-bit reference.

Tolerances as in the layer norm's own tests. A row is scaled by a power of two there, which rounds nothing; the saved mean
may be a subnormal float32, half of whose step is 2^-150.
"""
import numpy as np
import pytest
import torch

import step_ref as ref
from gpu_util import need_gpu, say
from test_gpu_norm import D, TYPES, _chain, _check, _ex, _vector

pytestmark = pytest.mark.gpu
COLS = [2, 3, 7, 8, 33, 64, 300, 700, 1500, 3000, 6000, 12000, 20000, 40000]
POWERS = (0, -50, -60, -62, -66, -70, -73, -75, -90, -100, -120, -126, -140)


def _rows(cols, dtype, seed=1):
    """Rows of every power of two, of mean 0 and of mean 20, and their values in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2 * len(POWERS), cols, generator=g, dtype=torch.float64)
    x[:, 0] += 0.5          # (no two equal values in the shortest rows)
    x[1::2] += 20
    x *= torch.tensor([2.0 ** k for k in POWERS for _ in range(2)], dtype=torch.float64)[:, None]
    x = x.float().to(TYPES[dtype])
    spread = x.double()
    some = ((spread - spread.mean(1, keepdim=True)) != 0).any(1)   # few bits may leave one value alone
    return x[some].cuda(), spread[some].numpy()


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 2.0 ** -122])
def test_small_rows(cols, dtype, wdtype, eps):
    hf = need_gpu()
    say("norm small", cols, dtype, wdtype, eps)
    xt, x = _rows(cols, dtype)
    wt, w = _vector(cols, wdtype, 4, 1.0)
    bt, b = _vector(cols, wdtype, 5, 0.0)
    want, mean, rstd, xh = ref.layer_norm(x, w, b, eps)
    y, saved = hf.layer_norm(xt, wt, bt, eps, save=True)
    _check(y, want, _ex(xh, cols) * np.abs(w) + D * (np.abs(xh * w) + np.abs(want)), dtype)
    assert torch.equal(hf.layer_norm(xt, wt, bt, eps), y)
    n = _chain(cols)
    _check(saved.mean[:, None], mean, D * n * np.abs(x - mean).mean(1, keepdims=True) + 2.0 ** -150, "f32")
    there = (rstd < 2.0 ** 127.9)[:, 0]
    _check(saved.rstd[:, None][torch.from_numpy(there).cuda()], rstd[there], D * (n / 2 + 8) * rstd[there], "f32")
    inside = hf.layer_norm(xt, wt, bt, eps, out=xt)
    assert inside is xt and torch.equal(xt, y)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -130, 2.0 ** -122])
def test_equal_small_values(cols, eps):
    """Nothing but eps is left: y is the bias, rstd that of eps."""
    hf = need_gpu()
    say("norm small equal", cols, eps)
    x = torch.tensor([0.0, 2.0 ** -149, 3e-42, -1e-36, 2.0 ** -80, 1.0], device="cuda")[:, None].repeat(1, cols)
    bt, _ = _vector(cols, "f32", 6, 0.0)
    y, saved = hf.layer_norm(x, None, bt, eps, save=True)
    assert torch.equal(y, bt.expand_as(y))
    assert torch.equal(saved.mean, x[:, 0])
    assert torch.allclose(saved.rstd.double(), torch.full((6,), eps ** -0.5, dtype=torch.float64, device="cuda"),
                          rtol=4 * D, atol=0)
