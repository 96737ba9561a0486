"""Layer norm at the ends of its range where a result is known to the bit, or to one rounding."""
import pytest
import torch

import step_ref as ref
from gpu_util import need_gpu, say
from test_gpu_norm import TYPES, _rows, _vector

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [3, 64, 700, 1500, 3000, 6000, 12000, 20000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dx_of_rows_beyond_float32(cols, dtype):
    """dx of a row times 2^k is the row's dx over 2^k. All operations on the scaled row are those on the row but for a power of
    two, so that only results below 2^-126 differ: there float32 and bfloat16 round to 2^-150 and 2^-134, while the row's
    own dx was rounded to its type."""
    hf = need_gpu()
    say("norm dx of large rows", cols, dtype)
    x, _ = _rows(5, cols, dtype, 7)
    powers = {1: 100, 3: 124}
    for row, k in powers.items():
        x[row] *= 2.0 ** k
    base = x.clone()
    for row, k in powers.items():
        base[row] *= 2.0 ** -k
    w, _ = _vector(cols, "f32", 8, 1.0)
    _, saved = hf.layer_norm(x, w, None, 0.0, save=True)
    _, plain = hf.layer_norm(base, w, None, 0.0, save=True)
    dy, _ = _rows(5, cols, dtype, 9)
    dx, dw, db = hf.layer_norm_backward(dy, x, saved, w)
    dz, ww, wb = hf.layer_norm_backward(dy, base, plain, w)
    assert torch.equal(dw, ww) and torch.equal(db, wb)      # xh and dy are the same
    least = 2.0 ** -150 + (2.0 ** -134 if dtype == "bf16" else 0.0)
    for row in range(5):
        k = powers.get(row, 0)
        got, want = dx[row].double() * 2.0 ** k, dz[row].double()
        small = got.abs() <= 2.0 ** (k - 126)
        assert torch.equal(got[~small], want[~small]), row
        assert (got - want).abs().le(2.0 ** k * least + ref.HALF[dtype] * want.abs()).all(), row
    assert (dx[1] != 0).any() and (dx[3] != 0).any()


@pytest.mark.parametrize("cols", [3, 5, 48, 513, 1000, 2731, 3000, 4095, 9000, 20000])
@pytest.mark.parametrize("value", [1000.1, 0.7, -1e10, 1e15, 1.1e19, -7e25, 2.0 ** 127, 3e38, 1e-30])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_values_give_the_bias(cols, value, dtype):
    """Exactly. The first mean is a chain of at most 41 additions and a division off, so that the values' difference from it
    is a multiple of their last place, 42 of them at most; the sum of 20000 such whole numbers, at most 840000, is exact in
    float32 in any order, and its mean is the difference itself, which is taken off."""
    hf = need_gpu()
    say("norm equal", cols, value, dtype)
    x = torch.full((3, cols), value, device="cuda").to(TYPES[dtype])
    b, _ = _vector(cols, dtype, 5, 0.0)
    y, saved = hf.layer_norm(x, None, b, save=True)
    assert torch.equal(y, b.expand_as(y))
    assert torch.equal(saved.mean, x[:, 0].float()) and saved.rstd.isfinite().all()
    dx, dw, db = hf.layer_norm_backward(torch.ones_like(x), x, saved)
    assert (dw == 0).all() and (db == 3).all()
