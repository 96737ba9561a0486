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


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_small_rows(cols, dtype):
    """Up to the largest rstd that a float32 holds (dy small enough for dx to be one too). xh is formed from the saved mean, which
    is D of it, and 2^-150 as a subnormal, off."""
    hf = need_gpu()
    say("norm small gradients", cols, dtype)
    g = torch.Generator().manual_seed(2)
    powers = (0, -60, -100, -120, -124, -126)
    x = torch.randn(3 * len(powers), cols, generator=g, dtype=torch.float64)
    x[:, 0] += 0.5
    # deviations of 1, 3/4 and 9/16: the last row's rstd is 2^126.8
    x = (x - x.mean(1, keepdim=True)) / x.std(1, keepdim=True, unbiased=False)
    x = x * torch.tensor([s * 2.0 ** k for k in powers for s in (1, 0.75, 0.5625)], dtype=torch.float64)[:, None]
    x[0] += 20
    xt = x.float().to(TYPES[dtype]).cuda()
    x = xt.double().cpu().numpy()
    gt = (torch.randn(len(x), cols, generator=g) * 2.0 ** -30).to(TYPES[dtype]).cuda()
    dy = gt.double().cpu().numpy()
    wt, w = _vector(cols, "f32", 4, 1.0)
    _, saved = hf.layer_norm(xt, wt, None, 0.0, save=True)
    _, mu, rstd, xh = ref.layer_norm(x, w, 0.0, 0.0)
    assert saved.rstd.isfinite().all() and rstd.max() > 2.0 ** 126.5
    dx, dw, db = hf.layer_norm_backward(gt, xt, saved, wt)
    n = _chain(cols)
    ex = _ex(xh, cols) + D * np.abs(mu) * rstd + 2 * D * np.abs(xh) + 2.0 ** -150 * rstd
    want, ww, wb = ref.layer_norm_grad(dy, xh, rstd, w)
    a = dy * w
    ma, mh = np.abs(a).mean(1, keepdims=True), np.abs(a * xh).mean(1, keepdims=True)
    pair = np.abs((a * xh).mean(1, keepdims=True))
    err = rstd * (D * (4 * np.abs(a) + (n + 4) * ma + np.abs(xh) * (n + 4) * mh)
                  + np.abs(xh) * (np.abs(a) * ex).mean(1, keepdims=True) + ex * pair)
    err = err + (n / 2 + 8) * D * np.abs(want) + 3 * D * np.abs(want)
    _check(dx, want, err, dtype)
    _check(dw, ww, (np.abs(dy) * ex).sum(0) + (len(x) + 2) * D * np.abs(dy * xh).sum(0), "f32")
    _check(db, wb, len(x) * D * np.abs(dy).sum(0), "f32")


@pytest.mark.parametrize("cols", [3, 64, 3000, 20000, 40000])
def test_gradients_of_the_largest_rstd(cols):
    """Rows of two values whose deviation is 2^-127.5: rstd is float32's last power of two and a half, xh is -1 and 1."""
    hf = need_gpu()
    say("norm small largest rstd", cols)
    d = round(2.0 ** 21.5) * 2.0 ** -149
    sign = torch.ones(cols, dtype=torch.float64)
    sign[:cols // 2] = -1.0
    if cols % 2:
        sign[-1] = 0.0
    xt = (sign * d).float()[None, :].repeat(5, 1).cuda()
    x = xt.double().cpu().numpy()
    g = torch.Generator().manual_seed(3)
    gt = (torch.randn(5, cols, generator=g) * 2.0 ** -30).cuda()
    dy = gt.double().cpu().numpy()
    _, saved = hf.layer_norm(xt, None, None, 0.0, save=True)
    _, mu, rstd, xh = ref.layer_norm(x, 1.0, 0.0, 0.0)
    assert (rstd > 2.0 ** 127.4).all() and saved.rstd.isfinite().all()
    dx, dw, db = hf.layer_norm_backward(gt, xt, saved)
    n = _chain(cols)
    ex = _ex(xh, cols) + 2 * D * np.abs(xh) + 2.0 ** -150 * rstd
    want, ww, _ = ref.layer_norm_grad(dy, xh, rstd, 1.0)
    ma, mh = np.abs(dy).mean(1, keepdims=True), np.abs(dy * xh).mean(1, keepdims=True)
    pair = np.abs((dy * xh).mean(1, keepdims=True))
    err = rstd * (D * (4 * np.abs(dy) + (n + 4) * ma + np.abs(xh) * (n + 4) * mh)
                  + np.abs(xh) * (np.abs(dy) * ex).mean(1, keepdims=True) + ex * pair)
    _check(dx, want, err + (n / 2 + 11) * D * np.abs(want), "f32")
    _check(dw, ww, (np.abs(dy) * ex).sum(0) + 7 * D * np.abs(dy * xh).sum(0), "f32")
