"""The linear layer on the GPU against a plain 64-bit reference.

Tolerances, derived: a float32 sum of n products is at most n 2^-23 sum |a b| off (each product's and each
addition's rounding, with a factor of two for the order); the activations' slope is at most 1.13, their own
error 2^-19 of their argument, the second derivative of each at most 1.13 too (silu's 0.5, gelu's 0.8); an output
is rounded to its type, at most half a step. dz is rounded once more, z before it.
"""
import numpy as np
import pytest
import torch

import step_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS, ACT = 2.0 ** -23, 2.0 ** -19


def _make(rows, cols, dtype, seed, scale=1.0, ld=None, offset=0):
    ld = ld or cols
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, ld), generator=g) * scale).to(TYPES[dtype])
    flat = torch.zeros(rows * ld + offset, dtype=x.dtype)
    flat[offset:] = x.reshape(-1)
    view = flat.cuda()[offset:].view(rows, ld)[:, :cols]
    return view, view.double()


def _check(got, want, err, dtype, name):
    got = got.double()
    bound = err + ref.HALF[dtype] * want.abs() + ref.TINY[dtype]
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (name, bad.nonzero()[:3], got[bad][:3], want[bad][:3], bound[bad][:3])


def _act(z, kind):
    """act and act' in float64, on the device."""
    if kind is None:
        return z, torch.ones_like(z)
    if kind == 0:
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if kind == 1:
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
    return z.clamp(min=0), (z > 0).double()


def _forward(hf, T, K, N, dtype, act, bias, res, lds, off):
    xt, x = _make(T, K, dtype, 1, 1.0, lds[0], off)
    wt, w = _make(N, K, dtype, 2, K ** -0.5, lds[1], off)
    bt, b = _make(1, N, dtype, 3)
    rt, r = _make(T, N, dtype, 4, 1.0, lds[3], off)
    bt = bt[0].contiguous() if bias else None
    out = torch.full((T * lds[2] + off,), 7.0, dtype=TYPES[dtype], device="cuda")[off:].view(T, lds[2])
    y, kept = hf.linear(xt, wt, bt, act, residual=rt if res else None, save=True, out=out[:, :N])
    assert y.data_ptr() == out.data_ptr() and (out[:, N:] == 7.0).all()
    z, ez = x @ w.T, (K + 1) * EPS * (x.abs() @ w.abs().T)
    if bias:
        z, ez = z + b, ez + EPS * (z + b).abs()
    a = _act(z, act)[0]
    want = a + r if res else a
    ea = ez if act is None else 1.13 * ez + ACT * z.abs()
    _check(y, want, ea + EPS * want.abs(), dtype, "y")
    if act is None:
        assert kept is None
    else:
        _check(kept, z, ez, dtype, "z")
    assert torch.equal(hf.linear(xt, wt, bt, act, residual=rt if res else None), y)
    return (xt, x), (wt, w), kept


def _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, off):
    (xt, x), (wt, w) = xs, ws
    gt, dy = _make(T, N, dtype, 5, 0.25, lds[2], off)
    dx, dw, db = hf.linear_backward(gt, xt, wt, z, act)
    dz, half = dy, torch.zeros_like(dy)
    if act is not None:
        dz = dy * _act(z.double(), act)[1]          # z as it was kept
        half = (ref.HALF[dtype] * dz.abs() + ref.TINY[dtype]) + ACT * (1 + z.double().abs()) * dy.abs()
    mag = dz.abs() + half
    _check(dx, dz @ w, half @ w.abs() + N * EPS * (mag @ w.abs()), dtype, "dx")
    _check(dw, dz.T @ x, half.T @ x.abs() + T * EPS * (mag.T @ x.abs()), dtype, "dw")
    exact = torch.zeros_like(dy) if act is None else ACT * (1 + z.double().abs()) * dy.abs()
    _check(db, dz.sum(0), exact.sum(0) + T * EPS * dz.abs().sum(0), dtype, "db")
    again = hf.linear_backward(gt, xt, wt, z, act)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))
    for asked in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        got = hf.linear_backward(gt, xt, wt, z, act, *asked)
        for need, a, b in zip(asked, got, (dx, dw, db)):
            assert (a is None) != need
            if need:   # another division of the work may add up in another order
                assert torch.allclose(a.double(), b.double(), rtol=4 * ref.HALF[dtype], atol=1e-3)


SHAPES = [  # T, K, N, (ldx, ldw, ldy, ldr), offset in elements
    (1, 1, 1, None, 0), (1, 64, 32, None, 0), (3, 40, 33, None, 0), (16, 72, 100, (80, 88, 104, 120), 0),
    (17, 72, 100, (80, 88, 104, 120), 0), (5, 37, 31, None, 1), (64, 128, 128, None, 0), (65, 136, 260, None, 8),
    (129, 200, 70, None, 1), (16, 256, 512, None, 0), (300, 96, 257, (99, 97, 301, 259), 3), (260, 520, 264, None, 0),
    (2, 1030, 96, None, 0), (40, 2048, 64, None, 0), (33, 64, 600, (64, 64, 602, 601), 0), (1, 4099, 65, None, 0),
    (7, 520, 4096, None, 0), (20, 5000, 40, None, 0), (200, 3001, 130, None, 0), (2, 63, 5, None, 0),
    (18, 1, 20, None, 0), (70, 8, 8, None, 0)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:3])))
@pytest.mark.parametrize("dtype,act,bias,res", [("bf16", None, True, True), ("f16", 1, True, False),
                                                ("bf16", 0, False, True), ("f16", 2, True, True),
                                                ("f16", None, False, False)])
def test_forward_and_backward(shape, dtype, act, bias, res):
    hf = need_gpu()
    T, K, N, lds, off = shape
    lds = lds or (K, K, N, N)
    say("linear", shape, dtype, act, bias, res)
    xs, ws, z = _forward(hf, T, K, N, dtype, act, bias, res, lds, off)
    _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, off)


@pytest.mark.parametrize("T,K,N", [(2048, 512, 2560), (4100, 264, 2056), (1000, 4096, 520), (8192, 136, 256),
                                   (100, 72, 20000), (30, 16400, 264), (17, 4096, 4096), (16, 11264, 1040),
                                   (1, 8192, 10000), (520, 1000, 2728), (3, 264, 70000)])
@pytest.mark.parametrize("dtype,act", [("bf16", None), ("f16", 0), ("bf16", 1)])
def test_many_tiles(T, K, N, dtype, act):
    """Sizes at which each kind of tile, and sums in parts, are chosen."""
    hf = need_gpu()
    say("linear tiles", T, K, N, dtype, act)
    lds = (K, K, N, N)
    xs, ws, z = _forward(hf, T, K, N, dtype, act, True, True, lds, 0)
    _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, 0)


@pytest.mark.parametrize("T,K,N", [(500, 2040, 4100), (260, 4104, 4000), (700, 16400, 264), (500, 1000, 1100),
                                   (2048, 512, 1400), (1000, 1027, 4000), (257, 72, 8200), (128, 4096, 11264),
                                   (30000, 100, 130), (250, 2050, 4000), (33, 4096, 11270), (100, 9000, 1100),
                                   (300, 2055, 2000), (48, 5000, 5001)])
@pytest.mark.parametrize("dtype,act,bias,res", [("bf16", 1, True, True), ("f16", None, False, True),
                                                ("bf16", 2, True, False)])
def test_a_workgroup_a_cu(T, K, N, dtype, act, bias, res):
    """Sizes whose tiles have four to eight stages, with steps that are no multiple of them, and in parts."""
    hf = need_gpu()
    say("linear deep", T, K, N, dtype, act, bias, res)
    lds = (K, K, N, N)
    xs, ws, z = _forward(hf, T, K, N, dtype, act, bias, res, lds, 0)
    _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, 0)


@pytest.mark.parametrize("T,K,N,lds,off", [(1000, 1026, 4000, None, 0), (2100, 4, 5000, None, 0), (4100, 70, 4100, None, 0),
                                           (300, 1998, 1030, None, 0), (520, 16414, 264, None, 0),
                                           (600, 2046, 1100, (2050, 2060, 1100, 1101), 2), (600, 2046, 1100, (2051, 2046, 1100, 1100), 0),
                                           (600, 2046, 1100, (2046, 2047, 1100, 1100), 0), (3000, 7, 3000, (8, 12, 3000, 3000), 0),
                                           (600, 2040, 1100, (2042, 2046, 1100, 1100), 6)])
@pytest.mark.parametrize("dtype,act", [("bf16", 1), ("f16", None)])
def test_rows_of_words_in_tiles(T, K, N, lds, off, dtype, act):
    """K that is no multiple of 8, rows and tensors at whole words but not at 16 bytes, one operand copied and one not."""
    hf = need_gpu()
    say("linear words", T, K, N, lds, off, dtype, act)
    lds = lds or (K, K, N, N)
    xs, ws, z = _forward(hf, T, K, N, dtype, act, True, True, lds, off)
    _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, off)


@pytest.mark.parametrize("T,K,N", [(1, 64, 40), (9, 1000, 300), (40, 264, 100), (300, 520, 520), (20, 8192, 64)])
@pytest.mark.parametrize("act", [None, 0])
def test_the_residual_may_be_the_output(T, K, N, act):
    hf = need_gpu()
    x, _ = _make(T, K, "bf16", 11)
    w, _ = _make(N, K, "bf16", 12, K ** -0.5)
    r, _ = _make(T, N, "bf16", 13, ld=N + 3)
    want = hf.linear(x, w, None, act, residual=r)
    assert hf.linear(x, w, None, act, residual=r, out=r) is r
    assert torch.equal(r, want)


@pytest.mark.parametrize("T,K,N", [(1, 64, 40), (40, 264, 100), (300, 520, 4096), (20, 8192, 64), (2100, 136, 2600),
                                   (500, 2040, 4104), (260, 4104, 4000)])
def test_z_without_an_activation(T, K, N):
    """The C call takes a z then, too: y before the residual."""
    import ctypes
    hf = need_gpu()
    x, _ = _make(T, K, "bf16", 30)
    w, _ = _make(N, K, "bf16", 31, K ** -0.5)
    b, r = _make(1, N, "bf16", 32)[0][0].contiguous(), _make(T, N, "bf16", 33)[0]
    y, z = torch.empty_like(r), torch.empty_like(r)
    d = hf.LinearDesc(T, K, N, K, K, N, N, 1, hf.GATE_NONE, 16)
    n = ctypes.c_int64()
    assert hf.lib().hobflops_linear_workspace(ctypes.byref(d), 0, ctypes.byref(n)) == 0
    ws = torch.empty(n.value + 16, dtype=torch.uint8, device="cuda")
    assert hf.lib().hobflops_linear(ctypes.byref(d), *[t.data_ptr() for t in (x, w, b, r, y, z, ws)], n.value,
                                    torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(z, hf.linear(x, w, b)) and torch.equal(y, hf.linear(x, w, b, residual=r))


@pytest.mark.parametrize("T,K,N", [(1, 96, 40), (5, 1000, 33), (40, 264, 100), (300, 520, 520), (20, 8192, 64),
                                   (2100, 136, 2600)])
@pytest.mark.parametrize("act", [None, 0, 1, 2])
def test_what_is_not_finite(T, K, N, act):
    """NaN and infinities of a token stay in its outputs, those of a row of w or of bias in theirs."""
    hf = need_gpu()
    x, _ = _make(T, K, "f16", 14)
    w, _ = _make(N, K, "f16", 15, K ** -0.5)
    b, _ = _make(1, N, "f16", 16)
    b = b[0].contiguous()
    r, _ = _make(T, N, "f16", 17)
    base = hf.linear(x, w, b, act, residual=r)
    x, w, b, r = x.clone(), w.clone(), b.clone(), r.clone()
    x[T - 1, K - 1] = float("nan")
    w[N - 2, 0] = float("inf")
    b[3] = float("nan")
    r[0, 5] = -float("inf")
    y = hf.linear(x, w, b, act, residual=r)
    same = torch.ones(T, N, dtype=torch.bool, device="cuda")
    same[T - 1], same[:, N - 2], same[:, 3], same[0, 5] = False, False, False, False
    assert torch.equal(y[same], base[same])
    assert y[T - 1].isnan().logical_or(torch.isinf(y[T - 1])).all() and y[:, 3].isnan().all()
    if T > 1:
        assert y[0, 5] == -float("inf")


def test_no_tokens():
    hf = need_gpu()
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), _make(40, 64, "bf16", 18)[0]
    y, z = hf.linear(x, w, act=hf.GATE_SILU, save=True)
    assert y.shape == z.shape == (0, 40)
    dx, dw, db = hf.linear_backward(y, x, w, z, hf.GATE_SILU)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("T,ld", [(3, (1 << 26) - 2), (40, (1 << 25) + 2), (40, 1 << 24)])
def test_rows_far_apart(T, ld):
    """Rows of x, y, dy and the residual whose offsets pass 31 bits."""
    hf = need_gpu()
    say("linear rows far apart", T, ld)
    K, N = 136, 200
    x, _ = _make(T, K, "bf16", 19)
    w, _ = _make(N, K, "bf16", 20, K ** -0.5)
    r, _ = _make(T, N, "bf16", 21)
    far = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)
    fx, fy, fr = far[:, :K], far[:, 512:512 + N], far[:, 1024:1024 + N]
    fx.copy_(x)
    fr.copy_(r)
    y, z = hf.linear(x, w, None, 0, residual=r, save=True)
    got, fz = hf.linear(fx, w, None, 0, residual=fr, save=True, out=fy)
    assert torch.equal(got, y) and torch.equal(fz, z)
    a = hf.linear_backward(fy, fx, w, z, 0)
    b = hf.linear_backward(y, x, w, z, 0)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_arguments():
    hf = need_gpu()
    x, w = _make(3, 64, "bf16", 22)[0], _make(40, 64, "bf16", 23)[0]
    y = hf.linear(x, w)
    with pytest.raises(hf.HobflopsError):
        hf.linear(x.float(), w.float())
    with pytest.raises(hf.HobflopsError):
        hf.linear(x, w, act=3)
    with pytest.raises(TypeError):
        hf.linear(x, w.half())
    with pytest.raises(ValueError):
        hf.linear(x, w[:, :63])
    with pytest.raises(ValueError):
        hf.linear(x[:, ::2], w[:, :32])
    with pytest.raises(ValueError):
        hf.linear(x, w, bias=y[0, :39])
    with pytest.raises(TypeError):
        hf.linear(x, w, bias=y[0].float())
    with pytest.raises(ValueError):
        hf.linear(x, w, residual=y[:2])
    with pytest.raises(ValueError):
        hf.linear(x, w, out=y[:2])
    with pytest.raises(ValueError):
        hf.linear_backward(y, x, w, None, hf.GATE_SILU)
    with pytest.raises(ValueError):
        hf.linear_backward(y[:2], x, w)
    assert hf.linear_backward(y, x, w, dx=False, dw=False, db=False) == (None, None, None)
