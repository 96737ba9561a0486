"""Layer norm on the GPU against a plain 64-bit reference.

Tolerance, derived, with d = 2^-24 (a float32 rounding) and n the longest chain of additions in a sum over
a row: 16 values of a thread (cols / 1024 of rows beyond 16384), 6 for the wave, 15 for the waves. A
sum is n d of its values' magnitudes off. Differences from the mean are d |x - mean| off and their mean, taken
off again, n d mean|x - mean|; the variance n d; rstd half of that and four roundings. So xh is off by
ex = d ((n / 2 + 8) |xh| + n + 2). With the saved mean, a float32, another d |mean| rstd. Everything
else is counted operation by operation, and doubled for products of errors.
"""
import numpy as np
import pytest
import torch

import step_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
D = 2.0 ** -24


def _rows(rows, cols, dtype, seed, ld=None, offset=0, scale=1.0, mean=0.0):
    """(GPU view of a wider, possibly misaligned tensor, float64 array)."""
    ld = ld or cols
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, ld), generator=g) * scale + mean).to(TYPES[dtype])
    flat = torch.zeros(rows * ld + offset, dtype=x.dtype)
    flat[offset:] = x.reshape(-1)
    view = flat.cuda()[offset:].view(rows, ld)[:, :cols]
    return view, view.double().cpu().numpy()


def _vector(cols, dtype, seed, mean):
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(cols, generator=g) / 4 + mean).to(TYPES[dtype])
    return v.cuda(), v.double().numpy()


def _chain(cols):
    return max(16, cols / 1024) + 21


def _ex(xh, cols):
    n = _chain(cols)
    return D * ((n / 2 + 8) * np.abs(xh) + n + 2)


def _check(got, want, err, dtype):
    got = got.double().cpu().numpy()
    bound = 2 * err + ref.HALF[dtype] * np.abs(want) + ref.TINY[dtype]
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], bound[bad][:3])


def _case(hf, rows, cols, dtype, wdtype, ld=None, off=0, scale=1.0, mean=0.0, eps=1e-5, add=True, affine=True):
    xt, x = _rows(rows, cols, dtype, 1, ld, off, scale, mean)
    gt, dy = _rows(rows, cols, dtype, 2, ld, off, 0.25)
    at, more = _rows(rows, cols, dtype, 3, ld, off, 0.25)
    wt, w = _vector(cols, wdtype, 4, 1.0) if affine else (None, 1.0)
    bt, b = _vector(cols, wdtype, 5, 0.0) if affine else (None, 0.0)
    out = torch.full((rows, cols + 3), 7.0, dtype=TYPES[dtype], device="cuda")
    y, saved = hf.layer_norm(xt, wt, bt, eps, save=True, out=out[:, :cols])
    want, mu, rstd, xh = ref.layer_norm(x, w, b, eps)
    ex = _ex(xh, cols)
    _check(y, want, ex * np.abs(w) + D * (np.abs(xh * w) + np.abs(want)), dtype)
    assert (out[:, cols:] == 7.0).all()
    assert torch.equal(hf.layer_norm(xt, wt, bt, eps), y)
    n = _chain(cols)
    _check(saved.mean[:, None], mu, D * n * np.abs(x - mu).mean(1, keepdims=True), "f32")
    _check(saved.rstd[:, None], rstd, D * (n / 2 + 8) * rstd, "f32")
    dx, dw, db = hf.layer_norm_backward(gt, xt, saved, wt, add=at if add else None)
    wdtype = wdtype if affine else dtype     # (without weight dw and db are of x's type)
    assert dw.dtype == db.dtype == TYPES[wdtype]
    more = more if add else 0.0
    want, ww, wb = ref.layer_norm_grad(dy, xh, rstd, w, more)
    ex = ex + D * np.abs(mu) * rstd + 2 * D * np.abs(xh)
    a = dy * w
    ma, mh = np.abs(a).mean(1, keepdims=True), np.abs(a * xh).mean(1, keepdims=True)
    pair = np.abs((a * xh).mean(1, keepdims=True))
    err = rstd * (D * (4 * np.abs(a) + (n + 4) * ma + np.abs(xh) * (n + 4) * mh)
                  + np.abs(xh) * (np.abs(a) * ex).mean(1, keepdims=True) + ex * pair)
    err = err + (n / 2 + 8) * D * np.abs(want - more) + 3 * D * (np.abs(want) + np.abs(more))
    _check(dx, want, err, dtype)
    # rows one after the other, in the worst order
    _check(dw, ww, (np.abs(dy) * ex).sum(0) + (rows + 2) * D * np.abs(dy * xh).sum(0), wdtype)
    _check(db, wb, rows * D * np.abs(dy).sum(0), wdtype)
    again = hf.layer_norm_backward(gt, xt, saved, wt, add=at if add else None)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))
    only = hf.layer_norm_backward(gt, xt, saved, wt, add=at if add else None, dw=False, db=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = hf.layer_norm_backward(gt, xt, saved, wt, add=at if add else None, db=False)
    assert torch.equal(only[1], dw) and only[2] is None
    only = hf.layer_norm_backward(gt, xt, saved, wt, add=at if add else None, dw=False)
    assert torch.equal(only[2], db) and only[1] is None


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2), (5, 7), (3, 8), (4, 33), (9, 64), (2, 511), (6, 512),
                                       (7, 513), (1, 1000), (13, 1024), (3, 1025), (5, 2048), (2, 2049),
                                       (4, 4096), (1, 4096), (3, 4097), (2, 8192), (3, 8193), (2, 16384),
                                       (3, 16385), (2, 40001), (300, 96), (130, 1030), (2, 12291)])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32"), ("bf16", "f32"),
                                          ("f16", "f16")])
def test_forward_and_backward(rows, cols, dtype, wdtype):
    hf = need_gpu()
    say("norm", rows, cols, dtype, wdtype)
    _case(hf, rows, cols, dtype, wdtype, add=rows % 2 == 0, affine=cols % 7 != 0)


@pytest.mark.parametrize("cols", [40, 1000, 2056, 2731, 5000, 9000, 16381, 17000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_apart_and_misaligned(cols, dtype):
    hf = need_gpu()
    say("norm apart", cols, dtype)
    _case(hf, 6, cols, dtype, "f32", ld=cols + 5, off=3)


@pytest.mark.parametrize("rows,cols", [(2100, 40), (9000, 17), (4200, 1100), (2500, 2100), (1100, 5000),
                                       (600, 9000), (2300, 16400)])
def test_more_rows_than_workgroups(rows, cols):
    hf = need_gpu()
    say("norm many rows", rows, cols)
    _case(hf, rows, cols, "bf16", "f32")


@pytest.mark.parametrize("rows,cols", [(5, 16385), (300, 17000), (3, 32768), (7, 32777), (4, 40001)])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_wide_rows(rows, cols, dtype, wdtype):
    """Four times 16 bytes a lane, and rows that are walked."""
    hf = need_gpu()
    say("norm wide", rows, cols, dtype, wdtype)
    _case(hf, rows, cols, dtype, wdtype)
    x, _ = _rows(rows, cols, dtype, 14, cols + 1, 1)
    want = hf.layer_norm(x)
    assert hf.layer_norm(x, out=x) is x and torch.equal(x, want)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (700, 3), (300000, 3), (262145, 5), (1000, 7), (64, 6)])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_rows_of_a_few_values(rows, cols, dtype, wdtype):
    hf = need_gpu()
    say("norm few", rows, cols, dtype, wdtype)
    _case(hf, rows, cols, dtype, wdtype, cols + 2, 1)
    x, _ = _rows(rows, cols, dtype, 15)
    want = hf.layer_norm(x)
    assert hf.layer_norm(x, out=x) is x and torch.equal(x, want)


@pytest.mark.parametrize("cols", [1, 2, 3, 7])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_few_large_and_odd_values(cols, dtype):
    hf = need_gpu()
    x, _ = _rows(6, cols, dtype, 16)
    x[1] *= 2.0 ** 100
    x[3, 0] = float("inf")
    x[4, cols - 1] = float("nan")
    base = x.clone()
    base[1] *= 2.0 ** -100
    y, saved = hf.layer_norm(x, eps=0.0 if cols > 1 else 1e-5, save=True)
    z = hf.layer_norm(base, eps=0.0 if cols > 1 else 1e-5)
    assert y[3].isnan().all() and y[4].isnan().all()
    for row in (0, 1, 2, 5):
        # (the quotient of two roundings' neighbours: a few steps)
        assert torch.allclose(y[row].double(), z[row].double(), rtol=0, atol=8 * ref.HALF[dtype])
    assert saved.rstd[1].isfinite() and saved.mean[1].isfinite()


@pytest.mark.parametrize("cols", [40, 20000, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_wide_values(cols, dtype):
    hf = need_gpu()
    x = torch.full((3, cols), 2.0 ** 120, device="cuda").to(TYPES[dtype])
    x[1] = 0.0
    y, saved = hf.layer_norm(x, save=True)
    assert (y == 0).all() and saved.rstd.isfinite().all()
    dx, dw, db = hf.layer_norm_backward(torch.ones_like(x), x, saved)
    assert (dx == 0).all() and (dw == 0).all() and (db == 3).all()


@pytest.mark.parametrize("cols", [96, 1536, 4096, 20000])
def test_rows_far_from_zero(cols):
    """A mean a thousand times the deviation: what float32 holds of the differences is there."""
    hf = need_gpu()
    say("norm far", cols)
    _case(hf, 4, cols, "f32", "f32", mean=1000.0)


@pytest.mark.parametrize("cols", [64, 3000, 20000])
@pytest.mark.parametrize("scale,eps", [(1e-3, 1e-5), (1e-6, 1e-5), (1e-6, 0.0), (1e15, 1e-5)])
def test_small_and_large_rows(cols, scale, eps):
    hf = need_gpu()
    say("norm scale", cols, scale, eps)
    _case(hf, 3, cols, "f32", "f32", scale=scale, eps=eps, add=False)


@pytest.mark.parametrize("cols", [64, 700, 1500, 3000, 6000, 12000, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_squares_beyond_float32(cols, dtype):
    """Rows of values up to 2^127, between ordinary ones: the same as of the row divided by 2^100."""
    hf = need_gpu()
    x, _ = _rows(5, cols, dtype, 7)
    x[1] *= 2.0 ** 100
    x[3] *= 2.0 ** 124
    base = x.clone()
    base[1] *= 2.0 ** -100
    base[3] *= 2.0 ** -124
    w, _ = _vector(cols, "f32", 8, 1.0)
    y, saved = hf.layer_norm(x, w, None, 0.0, save=True)
    z, plain = hf.layer_norm(base, w, None, 0.0, save=True)
    tol = 2 * (_chain(cols) + 12) * D
    # (both within the bound of the exact one)
    assert torch.allclose(y.double(), z.double(), rtol=tol + 2 * ref.HALF[dtype], atol=16 * tol)
    for row, k in ((1, 100), (3, 124)):
        assert torch.allclose(saved.mean[row].double() * 2.0 ** -k, plain.mean[row].double(), rtol=0, atol=4 * tol)
        assert torch.allclose(saved.rstd[row].double() * 2.0 ** k, plain.rstd[row].double(), rtol=tol + 2.0 ** -21)
    dy, _ = _rows(5, cols, dtype, 9)
    dx = hf.layer_norm_backward(dy, x, saved, w)[1]
    dz = hf.layer_norm_backward(dy, base, plain, w)[1]
    assert torch.isfinite(dx).all()
    # (rstd of the largest row is a subnormal float32: 2^-21 of it)
    assert torch.allclose(dx.double(), dz.double(), rtol=0, atol=5 * 5 * (2.0 ** -20 + 16 * tol))


@pytest.mark.parametrize("cols", [48, 1000, 2000, 4000, 20000])
def test_what_is_not_finite_stays_in_its_row(cols):
    hf = need_gpu()
    x, _ = _rows(6, cols, "bf16", 10)
    base, kept = hf.layer_norm(x, save=True)
    x = x.clone()
    x[1, 0], x[2, cols // 2], x[4, cols - 1] = float("nan"), float("inf"), -float("inf")
    y, saved = hf.layer_norm(x, save=True)
    for row in range(6):
        if row in (1, 2, 4):
            assert y[row].isnan().all()
        else:
            assert torch.equal(y[row], base[row])
    dy, _ = _rows(6, cols, "bf16", 11)
    dx, dw, db = hf.layer_norm_backward(dy, x, saved)
    want = hf.layer_norm_backward(dy, torch.where(torch.isfinite(x), x, torch.zeros_like(x)), kept)
    assert torch.equal(dx[0], want[0][0]) and torch.equal(dx[5], want[0][5])
    assert dx[1].isnan().all() and dw.isnan().all() and torch.equal(db, want[2])


def test_constant_rows():
    hf = need_gpu()
    x = torch.tensor([[3.0] * 40, [0.0] * 40], device="cuda")
    assert (hf.layer_norm(x) == 0).all()
    assert hf.layer_norm(x, eps=0.0).isnan().all()
    y, saved = hf.layer_norm(x, save=True)
    dy = torch.ones_like(x)
    dx, dw, db = hf.layer_norm_backward(dy, x, saved)
    assert (dx == 0).all() and (dw == 0).all() and (db == 2).all()


@pytest.mark.parametrize("cols", [5, 48, 1000, 3000, 9000, 20000])
@pytest.mark.parametrize("value", [1000.1, -1e10, 1e15, 1.1e19, -7e25, 2.0 ** 127, 3e38])
def test_equal_values_far_from_zero(cols, value):
    """Nothing is left of them but rounding: a mean is _chain() roundings off, the difference's own mean as many of
    it, and rstd is at most 2^22 over that mean."""
    hf = need_gpu()
    say("norm equal", cols, value)
    x = torch.full((3, cols), value, device="cuda")
    x[1] = torch.arange(cols, device="cuda") % 7
    y, saved = hf.layer_norm(x, save=True)
    assert (y[0].abs() <= _chain(cols) / 2).all() and torch.equal(y[0], y[2])
    assert torch.equal(y[1], hf.layer_norm(x[1:2])[0])
    assert abs(saved.mean[0].item() / x[0, 0].item() - 1) <= 2 * D and saved.rstd.isfinite().all()
    dx, dw, db = hf.layer_norm_backward(torch.ones_like(x), x, saved)
    assert dx.isfinite().all() and dw.isfinite().all() and (db == 3).all()


def test_no_rows_and_in_place():
    hf = need_gpu()
    w = torch.ones(64, device="cuda")
    x = torch.empty(0, 64, device="cuda")
    y, saved = hf.layer_norm(x, w, save=True)
    assert y.shape == (0, 64)
    dx, dw, db = hf.layer_norm_backward(x, x, saved, w)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()
    for cols in (64, 3000, 20000):
        x, _ = _rows(5, cols, "bf16", 12)
        want = hf.layer_norm(x)
        assert hf.layer_norm(x, out=x) is x and torch.equal(x, want)


def test_rows_beyond_31_bits():
    """Rows whose offsets pass 2^31 values."""
    hf = need_gpu()
    ld, rows, cols = (1 << 30) + 8, 4, 1000
    near, _ = _rows(rows, cols, "bf16", 13)
    wide = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)[:, :cols]
    wide.copy_(near)
    y, saved = hf.layer_norm(wide, save=True)
    assert torch.equal(y, hf.layer_norm(near))
    got = hf.layer_norm_backward(wide, wide, saved, add=wide)
    assert all(torch.equal(a, b) for a, b in zip(got, hf.layer_norm_backward(near, near, saved, add=near)))


def test_arguments():
    hf = need_gpu()
    x = torch.zeros(4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, saved = hf.layer_norm(x, w, save=True)
    with pytest.raises(TypeError):
        hf.layer_norm(x.double())
    with pytest.raises(TypeError):
        hf.layer_norm(x, w.half())
    with pytest.raises(TypeError):
        hf.layer_norm(x.half(), w.half(), w)
    with pytest.raises(TypeError):
        hf.layer_norm(x, w.cpu())
    with pytest.raises(ValueError):
        hf.layer_norm(x, w[:63])
    with pytest.raises(ValueError):
        hf.layer_norm(x[:, ::2])
    with pytest.raises(ValueError):
        hf.layer_norm(x, out=x[:3])
    with pytest.raises(hf.HobflopsError):
        hf.layer_norm(x, w, eps=-1.0)
    with pytest.raises(hf.HobflopsError):
        hf.layer_norm(torch.empty(4, 0, device="cuda"))
    with pytest.raises(ValueError):
        hf.layer_norm_backward(x[:3], x, saved, w)
    with pytest.raises(TypeError):
        hf.layer_norm_backward(x.half(), x, saved, w)
    with pytest.raises(ValueError):
        hf.layer_norm_backward(x, x, hf.NormSaved(saved.mean[:2], saved.rstd), w)
