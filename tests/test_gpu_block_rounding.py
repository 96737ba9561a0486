"""Unpacked values are the code's value times the scale, rounded once to the output's type: 4-bit codes
under float32 and bfloat16 scales, whose products need more bits than float32 has."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def _round(v, dtype):
    """float64 values to nearest even in a type, as float64."""
    if dtype == torch.float32:
        return v.astype(np.float32).astype(np.float64)
    if dtype == torch.float16:
        return v.astype(np.float16).astype(np.float64)
    # bfloat16: 8 bits of fraction with the hidden one, the smallest step 2^-133
    e = np.maximum(np.frexp(np.where(v == 0, 1.0, v))[1] - 8, -133)
    r = np.ldexp(np.rint(np.ldexp(v, -e)), e)
    return np.where(np.abs(r) >= 2.0 ** 128, np.copysign(np.inf, v), r)


def test_reference_rounding():
    """The reference's bfloat16 rounding, of float32 values, is torch's."""
    need_gpu()
    bits = np.random.default_rng(0).integers(0, 0x7F800000, 100000, dtype=np.uint32)
    v = bits.view(np.float32)
    want = torch.from_numpy(v.copy()).bfloat16().double().numpy()
    assert np.array_equal(_round(v.astype(np.float64), torch.bfloat16), want)


@pytest.mark.parametrize("cols", [512, 509])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low,high", [(-26, 14), (-149, -126), (-140, 127), (118, 127)])
def test_unpack4_rounds_once(low, high, scale, dtype, cols):
    hf = need_gpu()
    say("unpack4 rounds once", low, high, scale, dtype, cols)
    rng = np.random.default_rng(low + 1000)
    rows, groups = 4096, 16
    # scales whose product by 1.5 and 3 falls on and beside the types' midpoints, and any others
    s = np.ldexp(1.0 + rng.random((rows, groups)), rng.integers(low, high, (rows, groups)))
    mid = rng.random((rows, groups)) < 0.7
    e = np.frexp(s)[1]
    m = np.rint(np.ldexp(s, 9 - e)) if dtype == torch.bfloat16 else np.rint(np.ldexp(s, 12 - e))
    n = np.ldexp(m, e - (9 if dtype == torch.bfloat16 else 12))
    near = (n / 1.5).astype(np.float32).astype(np.float64)
    s = torch.from_numpy(np.where(mid, near, s)).to(scale)
    f = s.double().numpy()
    packed = rng.integers(0, 256, (rows, (cols + 1) // 2), dtype=np.uint8)
    got = hf.block_unpack(torch.from_numpy(packed).cuda(), s.cuda(), cols, (2, 1), dtype=dtype)
    want = _round(ref.unpack(ref.nibbles(packed, cols), f, (2, 1)), dtype)
    got = got.double().cpu().numpy()
    assert np.array_equal(got, want)
    assert np.array_equal(np.signbit(got), np.signbit(want))


def test_unpack4_other_scales():
    """Scales of zero, infinity and NaN, and negative ones."""
    hf = need_gpu()
    s = torch.tensor([[0.0, -0.0, float("inf"), float("nan"), -1.3, -2.0 ** -149]])
    # every code in both halves of a byte, under each scale
    packed = np.tile(np.arange(16, dtype=np.uint8) | (15 - np.arange(16, dtype=np.uint8)) << 4, 6).reshape(1, 96)
    with np.errstate(invalid="ignore"):
        exact = ref.unpack(ref.nibbles(packed, 192), s.double().numpy(), (2, 1))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got = hf.block_unpack(torch.from_numpy(packed).cuda(), s.cuda(), 192, (2, 1), dtype=dtype)
        with np.errstate(invalid="ignore"):
            want = np.where(np.isfinite(exact), _round(np.nan_to_num(exact), dtype), exact)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
