"""Refusals of the layer norm, linear and AdamW entry points (CPU: no call reaches the GPU), the device a call
runs on, and the references' own checks."""
import ctypes

import numpy as np
import pytest
import torch

import narrow_ref
import step_ref as ref
from test_abi import FAKE, hf  # noqa: F401  (the library, as a fixture)
from test_devices import Gpu, _gpu, calls  # noqa: F401

ODD = ctypes.c_void_p(0x10001)
BIG = 1 << 40


def _norm_desc(hf, **kw):
    d = dict(rows=4, cols=64, ldx=64, ldy=64, ld_add=64, type=1, wtype=0, eps=1e-5)
    d.update(kw)
    return ctypes.byref(hf.NormDesc(*d.values()))


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), -1), (dict(cols=0), -1), (dict(ldx=63), -1), (dict(ldy=63), -1), (dict(type=3), -1),
    (dict(wtype=3), -1), (dict(wtype=2), -2), (dict(type=0, wtype=1), -2), (dict(eps=-1e-9), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(rows=1 << 40), -1),
    (dict(cols=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), -1)])
def test_norm_refusals(hf, bad, status):
    L, n = hf.lib(), ctypes.c_int64()
    d = _norm_desc(hf, **bad)
    assert L.hobflops_layer_norm(d, *[FAKE] * 6, None) == status
    assert L.hobflops_layer_norm_workspace(d, ctypes.byref(n)) == status
    assert L.hobflops_layer_norm_backward(d, *[FAKE] * 10, BIG, None) == status


def test_norm_pointers(hf):
    L, n, d = hf.lib(), ctypes.c_int64(), _norm_desc(hf)
    assert L.hobflops_layer_norm(None, *[FAKE] * 6, None) == -1
    assert L.hobflops_layer_norm_workspace(d, None) == -1
    for i, status in ((0, -1), (3, -1), (4, -1), (5, -1)):   # x, y, mean and rstd
        args = [FAKE] * 6
        args[i] = None
        assert L.hobflops_layer_norm(d, *args, None) == status, i
    for i in range(6):
        args = [FAKE] * 6
        args[i] = ODD
        assert L.hobflops_layer_norm(d, *args, None) == -3, i
    assert L.hobflops_layer_norm(_norm_desc(hf, rows=0), *[None] * 6, None) == 0
    assert L.hobflops_layer_norm_workspace(d, ctypes.byref(n)) == 0 and n.value > 0
    assert L.hobflops_layer_norm_backward(d, *[FAKE] * 10, n.value - 1, None) == -1
    for i in (0, 1, 3, 4, 6, 9):                             # dy, x, mean, rstd, dx and the workspace
        args = [FAKE] * 10
        args[i] = None
        assert L.hobflops_layer_norm_backward(d, *args, BIG, None) == -1, i
    for i in range(10):
        args = [FAKE] * 10
        args[i] = ODD
        assert L.hobflops_layer_norm_backward(d, *args, BIG, None) == -3, i
    assert L.hobflops_layer_norm_backward(_norm_desc(hf, ld_add=63), *[FAKE] * 10, BIG, None) == -1


@pytest.mark.parametrize("y,kw", [
    (0x10002, {}), (0x10000 - 2 * 255, {}), (0x10000 + 2 * 255, {}),    # one value of the first or the last row
    (0x10000, dict(ldx=128)), (0x10000 + 2 * 65, dict(ldx=128, ldy=128)), (0x10000 + 2 * 64, dict(ldx=128, ldy=129)),
    (0x10000 + 2 * 64, dict(rows=1, cols=65, ldx=65, ldy=65)), (0x20000 - 2, {}), (0x30000 + 4 * 63, {})])
def test_norm_overlaps(hf, y, kw):
    """x at 0x10000, weight and bias (float32) at 0x20000 and 0x30000."""
    args = [ctypes.c_void_p(p) for p in (0x10000, 0x20000, 0x30000, y)]
    assert hf.lib().hobflops_layer_norm(_norm_desc(hf, **kw), *args, None, None, None) == -1


@pytest.mark.parametrize("kw", [
    dict(y=0x100000), dict(y=0x200000 + 2 * 64 * 95), dict(y=0x300000 - 2), dict(y=0x400002),
    dict(y=0x400000, ldr=97), dict(z=0x400000), dict(z=0x100000 - 2), dict(y=0x600000 + 2 * 96 * 19),
    dict(y=0x100000 + 2 * 63, ldx=192, ldy=192)])
def test_linear_overlaps(hf, kw):
    a = dict(x=0x100000, w=0x200000, bias=0x300000, residual=0x400000, y=0x500000, z=0x600000)
    d = _linear_desc(hf, **{k: v for k, v in kw.items() if k not in a})
    a.update({k: v for k, v in kw.items() if k in a})
    assert hf.lib().hobflops_linear(d, *[ctypes.c_void_p(p) for p in a.values()], FAKE, BIG, None) == -1


@pytest.mark.parametrize("kw", [dict(dx=0x100000), dict(dx=0x200000 + 2 * 255), dict(dx=0x600000 - 2), dict(dw=0x700000 + 4),
                                dict(dw=0x300000), dict(db=0x400000 - 4), dict(db=0x800000 + 4 * 63), dict(dw=0x500000)])
def test_norm_backward_overlaps(hf, kw):
    """dy, x (bfloat16), weight, mean, rstd (float32), add; dx, dw, db."""
    a = dict(dy=0x100000, x=0x200000, w=0x300000, mean=0x400000, rstd=0x500000, add=0x600000, dx=0x700000, dw=0x800000,
             db=0x900000, ws=0xa00000)
    a.update(kw)
    assert hf.lib().hobflops_layer_norm_backward(_norm_desc(hf), *[ctypes.c_void_p(p) for p in a.values()], BIG, None) == -1


@pytest.mark.parametrize("kw", [dict(dx=0x100000), dict(dx=0x200000), dict(dw=0x300000), dict(db=0x400000), dict(dw=0x500000 + 2),
                                dict(db=0x600000 + 2 * 64 * 95)])
def test_linear_backward_overlaps(hf, kw):
    a = dict(dy=0x100000, x=0x200000, w=0x300000, z=0x400000, dx=0x500000, dw=0x600000, db=0x700000, ws=0x800000)
    a.update(kw)
    assert hf.lib().hobflops_linear_backward(_linear_desc(hf), *[ctypes.c_void_p(p) for p in a.values()], BIG, None) == -1


def _linear_desc(hf, **kw):
    d = dict(T=20, K=64, N=96, ldx=64, ldw=64, ldy=96, ldr=96, type=1, act=0, align=16)
    d.update(kw)
    return ctypes.byref(hf.LinearDesc(*d.values()))


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), -1), (dict(K=0), -1), (dict(N=0), -1), (dict(ldx=63), -1), (dict(ldw=63), -1),
    (dict(ldy=95), -1), (dict(type=0), -2), (dict(type=5), -1), (dict(act=3), -1), (dict(act=-2), -1),
    (dict(align=0), -1), (dict(align=32), -1), (dict(T=1 << 25), -1), (dict(K=1 << 21, ldx=1 << 21, ldw=1 << 21), -1),
    (dict(N=1 << 21, ldy=1 << 21), -1)])
def test_linear_refusals(hf, bad, status):
    L, n = hf.lib(), ctypes.c_int64()
    d = _linear_desc(hf, **bad)
    assert L.hobflops_linear(d, *[FAKE] * 7, BIG, None) == status
    assert L.hobflops_linear_workspace(d, 0, ctypes.byref(n)) == status
    assert L.hobflops_linear_workspace(d, 7, ctypes.byref(n)) == status
    assert L.hobflops_linear_backward(d, *[FAKE] * 8, BIG, None) == status


def test_linear_pointers(hf):
    L, n, d = hf.lib(), ctypes.c_int64(), _linear_desc(hf)
    for need in (-1, 8):
        assert L.hobflops_linear_workspace(d, need, ctypes.byref(n)) == -1
    assert L.hobflops_linear_workspace(d, 0, None) == -1
    for i in (0, 1, 4):                                      # x, w, y
        args = [FAKE] * 7
        args[i] = None
        assert L.hobflops_linear(d, *args, BIG, None) == -1, i
    for i in range(6):
        args = [FAKE] * 7
        args[i] = ODD
        assert L.hobflops_linear(d, *args, BIG, None) == -3, i
    assert L.hobflops_linear(_linear_desc(hf, ldr=95), *[FAKE] * 7, BIG, None) == -1
    assert L.hobflops_linear(_linear_desc(hf, T=0), *[None] * 7, 0, None) == 0
    loose = _linear_desc(hf, T=4096, K=4096, N=4096, ldx=4096, ldw=4096, ldy=4096, ldr=4096, align=2)
    assert L.hobflops_linear_workspace(loose, 0, ctypes.byref(n)) == 0 and n.value > 0
    assert L.hobflops_linear(loose, *[FAKE] * 7, n.value - 1, None) == -1
    assert L.hobflops_linear(loose, *[FAKE] * 6, None, BIG, None) == -1
    assert L.hobflops_linear_workspace(d, 7, ctypes.byref(n)) == 0 and n.value > 0
    assert L.hobflops_linear_backward(d, *[FAKE] * 8, n.value - 1, None) == -1
    for i in (0, 1, 2, 3, 7):                                # dy, x, w, z and the workspace
        args = [FAKE] * 8
        args[i] = None
        assert L.hobflops_linear_backward(d, *args, BIG, None) == -1, i
    for i in range(8):
        args = [FAKE] * 8
        args[i] = ODD
        assert L.hobflops_linear_backward(d, *args, BIG, None) == -3, i
    assert L.hobflops_linear_backward(d, *[FAKE] * 4, None, None, None, FAKE, BIG, None) == -1


def _step(hf, tensors=((0x100000, 0x200000, 0x300000, 64),), m=0x400000, ms=0x500000, v=0x600000, vs=0x700000,
          length=64, desc=True, **kw):
    d = dict(grad_type=1, copy_type=2, states=hf.Fmt(4, 3), lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
             weight_decay=0.0, grad_scale=1.0, step=1, seed=0, lr_at=None, step_at=None, grad_scale_at=None,
             skip_at=None)
    d.update(kw)
    t = (hf.AdamwTensor * max(1, len(tensors)))(*[hf.AdamwTensor(*t) for t in tensors])
    return hf.lib().hobflops_adamw(ctypes.byref(hf.AdamwDesc(*d.values())) if desc else None, t, len(tensors),
                                   m, ms, v, vs, length, None)


T0 = (0x100000, 0x200000, 0x300000, 64)


@pytest.mark.parametrize("bad,status", [
    (dict(grad_type=3), -1), (dict(copy_type=0), -1), (dict(copy_type=3), -1), (dict(states=(0, 3)), -1),
    (dict(states=(2, 1)), -2), (dict(states=(5, 3)), -2), (dict(beta1=1.0), -1), (dict(beta1=-0.1), -1),
    (dict(beta2=1.0), -1), (dict(beta2=float("nan")), -1), (dict(eps=-1.0), -1), (dict(step=0), -1),
    (dict(length=63), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(ms=None), -1), (dict(vs=None), -1),
    (dict(desc=False), -1), (dict(lr_at=0x800001), -3), (dict(step_at=0x800004), -3), (dict(skip_at=0x800002), -3),
    (dict(tensors=((None, 0x200000, 0, 64),)), -1), (dict(tensors=((0x100002, 0x200000, 0, 64),)), -3),
    (dict(tensors=((0x100000, 0x200001, 0, 64),)), -3), (dict(tensors=((0x100000, 0x200000, 0x300001, 64),)), -3),
    (dict(tensors=((0x100000, 0x200000, 0, -1),)), -1), (dict(tensors=(T0, T0), length=128), -1),
    (dict(tensors=(T0, (0x1000fc, 0x210000, 0, 64)), length=128), -1),    # the last value of the first
    (dict(tensors=((0x100000, 0x100010, 0, 64),)), -1), (dict(tensors=((0x100000, 0x200000, 0x200010, 64),)), -1),
    (dict(m=0x100000), -1), (dict(v=0x400010), -1), (dict(ms=0x600000), -1), (dict(lr_at=0x100000), -1)])
def test_adamw_refusals(hf, bad, status):
    if "states" in bad:
        bad["states"] = hf.Fmt(*bad["states"])
    assert _step(hf, **bad) == status


def test_adamw_nothing_to_do(hf):
    assert _step(hf, tensors=(), m=None, v=None, length=0) == 0
    assert _step(hf, tensors=((None, None, None, 0),), m=None, v=None, length=0) == 0
    n = ctypes.c_int64()
    t = (hf.AdamwTensor * 3)(*[hf.AdamwTensor(None, None, None, k) for k in (1, 0, 33)])
    assert hf.lib().hobflops_adamw_state_len(t, 3, ctypes.byref(n)) == 0 and n.value == 96
    assert hf.lib().hobflops_adamw_state_len(t, 3, None) == -1
    t[1].n = -1
    assert hf.lib().hobflops_adamw_state_len(t, 3, ctypes.byref(n)) == -1


def test_host_tensors_are_refused(hf):
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        hf.layer_norm(x)
    with pytest.raises(TypeError):
        hf.linear(x, x)
    with pytest.raises(TypeError):
        hf.adamw([x], [x], hf.AdamWState(x, x, None), 1)


@pytest.mark.parametrize("current", [0, 1])
def test_a_call_runs_on_its_tensors_device(calls, monkeypatch, current):
    from paper_2007_06563_amd import hobflops as hf
    monkeypatch.setattr(hf, "_get_device", lambda t: t.device.index)
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **k: zeros(*a, **k).as_subclass(Gpu))
    f32 = torch.float32
    calls.device = current
    x = _gpu(4, 64)
    y, saved = hf.layer_norm(x, _gpu(64), save=True)
    hf.layer_norm_backward(y, x, saved, _gpu(64))
    y, z = hf.linear(x, _gpu(96, 64), _gpu(96), hf.GATE_SILU, save=True)
    hf.linear_backward(y, x, _gpu(96, 64), z, hf.GATE_SILU)
    p = [_gpu(40, dtype=f32), _gpu(8, dtype=f32)]
    for fmt in (None, (4, 3)):
        hf.adamw(p, [_gpu(40), _gpu(8)], hf.adamw_state(p, fmt), 1)
    names = [n for n, _, _ in calls.seen if "workspace" not in n]
    assert names == ["hobflops_layer_norm", "hobflops_layer_norm_backward", "hobflops_linear",
                     "hobflops_linear_backward", "hobflops_adamw", "hobflops_adamw"]
    assert all(d == 1 and s == 1001 for n, d, s in calls.seen if "workspace" not in n), calls.seen
    assert calls.device == current


# ---- the references' own checks ------------------------------------------------


def test_reference_gradients_by_differences():
    rng = np.random.default_rng(1)
    x, dy, w, b = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7)
    loss = lambda x, w, b: (ref.layer_norm(x, w, b, 1e-5)[0] * dy).sum()  # noqa: E731
    _, _, rstd, xh = ref.layer_norm(x, w, b, 1e-5)
    h = 1e-6
    for got, i in zip(ref.layer_norm_grad(dy, xh, rstd, w), range(3)):
        args = [x, w, b]
        for at in np.ndindex(args[i].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[i][at] += h
            down[i][at] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - got[at]) < 1e-7


@pytest.mark.parametrize("kind", [None, 0, 1, 2])
def test_reference_linear_gradients_by_differences(kind):
    rng = np.random.default_rng(2)
    x, w, b, r, dy = (rng.standard_normal(s) for s in ((3, 5), (4, 5), (4,), (3, 4), (3, 4)))
    loss = lambda x, w, b, r: ((ref.act(x @ w.T + b, kind)[0] + r) * dy).sum()  # noqa: E731
    dz = dy * ref.act(x @ w.T + b, kind)[1]
    h = 1e-6
    for got, i in zip((dz @ w, dz.T @ x, dz.sum(0), dy), range(4)):
        args = [x, w, b, r]
        for at in np.ndindex(args[i].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[i][at] += h
            down[i][at] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - got[at]) < 1e-7


def test_reference_step_is_the_formula():
    """The float32 reference against the formula in 64 bits: some roundings of each value apart."""
    rng = np.random.default_rng(3)
    n = 1000
    p, g = rng.standard_normal(n), rng.standard_normal(n) * 1e-3
    m, v = rng.standard_normal(n) * 1e-3, rng.random(n) * 1e-6
    p, g, m, v = (a.astype(np.float32) for a in (p, g, m, v))
    q, m2, v2, _ = ref.adamw(p, g, m, v, 7, 1e-2, (0.9, 0.999), 1e-8, 0.1, 0.5)
    d = g.astype(float) * 0.5
    m3, v3 = 0.9 * m.astype(float) + 0.1 * d, 0.999 * v.astype(float) + 0.001 * d * d
    step = 1e-2 / (1 - 0.9 ** 7) * m3 / (np.sqrt(v3 / (1 - 0.999 ** 7)) + 1e-8)
    want = p * (1 - 1e-2 * 0.1) - step
    mag = 0.9 * np.abs(m) + 0.1 * np.abs(d)
    assert (np.abs(m2 - m3) <= 5 * 2.0 ** -24 * mag).all() and (np.abs(v2 / v3 - 1) <= 6 * 2.0 ** -24).all()
    moved = 1e-2 / (1 - 0.9 ** 7) * mag / np.sqrt(v3 / (1 - 0.999 ** 7))
    assert (np.abs(q - want) <= 2.0 ** -24 * (4 * np.abs(p) + 16 * moved)).all()


@pytest.mark.parametrize("f", [(4, 3), (5, 2)])
def test_reference_rounding_keeps_the_means(f):
    """Over all numbers u a value's mean is itself, a root's mean square its square, within the distance of
    the numbers (2^-16 of a step); a root that is not 0 is never 0."""
    u = ((np.arange(65536) + 0.5) / 65536).astype(np.float32)
    top = narrow_ref.code_values(f)[-1]
    for x in (0.3, 1.0, 7.77, 100.1, 1e-3, 5e-7):
        row = np.zeros((65536, 32), np.float32)
        row[:, 0], row[:, 1] = top, x
        flat, noise = row.ravel(), u.repeat(32)
        _, k, q = ref.encode(flat, noise, f)
        got = (q.reshape(-1, 32)[:, 1].astype(float) * np.exp2(k.astype(float)))
        least = narrow_ref.code_values(f)[1]
        step = max(least, 2.0 ** (np.floor(np.log2(x)) - f[1]))
        assert abs(got.mean() - np.float32(x)) <= 2.0 ** -16 * step
        _, k, q = ref.encode(flat, noise, f, (row * row).ravel())
        r = (q.reshape(-1, 32)[:, 1].astype(float) * np.exp2(k.astype(float)))
        assert (r > 0).all()
        if x > least:
            # (float32 squares: 2^-22 of the upper one)
            assert abs((r * r).mean() - float(np.float32(x)) ** 2) <= (2.0 ** -16 * 2 * step + 2.0 ** -22 * (x + step)) * (x + step)


def test_reference_numbers_are_spread():
    """A counter's numbers: each bit, and its change with every bit of place, step and seed, a half."""
    n = 1 << 16
    um, ur = ref.uniform(np.arange(n), 5, 9)
    for u in (um, ur):
        # mean and mean square of n uniform numbers, to five deviations
        assert abs(u.mean() - 0.5) < 5 * (1 / 12 / n) ** 0.5 and abs((u.astype(float) ** 2).mean() - 1 / 3) < 5 * (4 / 45 / n) ** 0.5
        assert abs(np.corrcoef(u[1:], u[:-1])[0, 1]) < 5 / n ** 0.5
    assert abs(np.corrcoef(um, ur)[0, 1]) < 5 / n ** 0.5
    for other in ((6, 9), (5, 8), (5, 9 + (1 << 40)), (5 + (1 << 33), 9)):
        vm, vr = ref.uniform(np.arange(n), *other)
        assert abs(np.corrcoef(um, vm)[0, 1]) < 5 / n ** 0.5 and abs(np.corrcoef(ur, vr)[0, 1]) < 5 / n ** 0.5
    far, _ = ref.uniform(np.arange(n, dtype=np.uint64) + np.uint64(1 << 33), 5, 9)
    assert abs(np.corrcoef(um, far)[0, 1]) < 5 / n ** 0.5


def test_reference_state_follows_its_mean():
    """v in 8 bits under a steady gradient: after thousands of steps its mean over many values is the
    gradient's square, where rounding to nearest would have stopped it on the way."""
    rng = np.random.default_rng(4)
    n, f, beta = 32 * 64, (4, 3), 0.99
    g2 = (np.exp2(rng.uniform(-4, 0, n)) ** 2).astype(np.float32)
    r = np.zeros(n, np.float32)
    for step in range(1, 801):
        v = (r * r * np.float32(beta) + g2 * np.float32(1 - beta)).astype(np.float32)
        _, k, q = ref.encode(np.sqrt(v), ref.uniform(np.arange(n), step, 0)[1], f, v)
        r = q * np.ldexp(np.float32(1), k).astype(np.float32).repeat(32)
    share = (r.astype(float) ** 2 / g2).mean()
    # a step's variance is at most (1 - beta) of a code's step (a quarter of v), so that of v settles at an
    # eighth: the mean of n values, over 100 steps' memory, is within 5 sqrt(1 / 8 / n)
    assert abs(share - (1 - beta ** 800)) < 5 * (1 / 8 / n) ** 0.5
