"""Refusals of the block, gated and 4-bit entry points (CPU: no call reaches the GPU), and the
references' own checks."""
import ctypes

import numpy as np
import pytest

import narrow_ref as ref
from test_abi import FAKE, hf  # noqa: F401  (the library, as a fixture)

ODD = ctypes.c_void_p(0x10001)


def _pack(hf, src=FAKE, type=1, rows=4, cols=64, ld=64, f=(4, 3), group=32, scale=0, codes=FAKE,
          scales=FAKE):
    return hf.lib().hobflops_block_pack(src, type, rows, cols, ld, hf.fmt(f), group, scale, codes,
                                        scales, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), -1), (dict(cols=-1), -1), (dict(ld=63), -1), (dict(type=3), -1),
    (dict(type=-1), -1), (dict(group=16), -1), (dict(group=0), -1), (dict(scale=3), -1),
    (dict(scale=-1), -1), (dict(f=(0, 3)), -1), (dict(f=(5, 3)), -2), (dict(f=(3, 4)), -2),
    (dict(group=64), -2), (dict(scale=1), -2), (dict(src=None), -1), (dict(codes=None), -1),
    (dict(scales=None), -1), (dict(src=ODD), -3), (dict(rows=1 << 40), -1),
    (dict(cols=1 << 31, ld=1 << 31), -1), (dict(f=(2, 1), scale=2, scales=ODD), -3)])
def test_block_refusals(hf, bad, status):
    assert _pack(hf, **bad) == status
    a = dict(src=FAKE, type=1, rows=4, cols=64, ld=64, f=(4, 3), group=32, scale=0, codes=FAKE,
             scales=FAKE)
    a.update(bad)
    assert hf.lib().hobflops_block_unpack(a["codes"], a["scales"], a["rows"], a["cols"],
                                          hf.fmt(a["f"]), a["group"], a["scale"], a["src"],
                                          a["type"], a["ld"], None) == status


def test_block_nothing_to_do(hf):
    assert _pack(hf, rows=0, src=None, codes=None, scales=None) == 0
    assert _pack(hf, cols=0, ld=0, src=None, codes=None, scales=None) == 0


def _gated(hf, **kw):
    d = dict(T=4, D=64, F=96, ldx=64, ldw=64, ldh=96, type=1, act=0, ckpt=hf.fmt((4, 3)), align=16)
    d.update({k: v for k, v in kw.items() if k in d})
    return hf.GatedDesc(*d.values())


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), -1), (dict(D=0), -1), (dict(F=0), -1), (dict(ldx=63), -1), (dict(ldw=63), -1),
    (dict(ldh=95), -1), (dict(type=0), -2), (dict(type=5), -1), (dict(act=3), -1),
    (dict(act=-1), -1), (dict(align=0), -1), (dict(align=32), -1), (dict(T=1 << 25), -1), (dict(D=1 << 21, ldx=1 << 21, ldw=1 << 21), -1)])
def test_gated_refusals(hf, bad, status):
    L, n = hf.lib(), ctypes.c_int64()
    d = _gated(hf, **bad)
    for backward in (0, 1):
        assert L.hobflops_gated_workspace(ctypes.byref(d), backward, ctypes.byref(n)) == status
    assert L.hobflops_gated_forward(ctypes.byref(d), *[FAKE] * 9, 1 << 40, None) == status
    assert L.hobflops_gated_backward(ctypes.byref(d), *[FAKE] * 13, 1 << 40, None) == status


def test_gated_formats_pointers_and_workspace(hf):
    L, n = hf.lib(), ctypes.c_int64()
    for f, status in (((5, 3), -2), ((2, 1), -2), ((0, 3), -1)):
        d = _gated(hf, ckpt=hf.fmt(f))
        assert L.hobflops_gated_forward(ctypes.byref(d), *[FAKE] * 9, 1 << 40, None) == status
        assert L.hobflops_gated_backward(ctypes.byref(d), *[FAKE] * 13, 1 << 40, None) == status
    none = _gated(hf, ckpt=hf.fmt((0, 0)))
    assert L.hobflops_gated_backward(ctypes.byref(none), *[FAKE] * 13, 1 << 40, None) == -1
    d = _gated(hf)
    assert L.hobflops_gated_workspace(ctypes.byref(d), 0, None) == -1
    assert L.hobflops_gated_workspace(None, 0, ctypes.byref(n)) == -1
    assert L.hobflops_gated_workspace(ctypes.byref(d), 1, ctypes.byref(n)) == 0 and n.value > 0
    assert L.hobflops_gated_backward(ctypes.byref(d), *[FAKE] * 13, n.value - 1, None) == -1
    for i in range(13):
        args = [FAKE] * 13
        args[i] = None
        assert L.hobflops_gated_backward(ctypes.byref(d), *args, 1 << 40, None) == -1, i
    for i in range(8):
        args = [FAKE] * 9
        args[i] = None
        assert L.hobflops_gated_forward(ctypes.byref(d), *args, 1 << 40, None) == -1, i
    for i in (0, 1, 2, 3):
        args = [FAKE] * 9
        args[i] = ODD
        assert L.hobflops_gated_forward(ctypes.byref(d), *args, 1 << 40, None) == -3, i
    for i in (0, 7, 8, 9, 10, 11, 12):
        args = [FAKE] * 13
        args[i] = ODD
        assert L.hobflops_gated_backward(ctypes.byref(d), *args, 1 << 40, None) == -3, i
    empty = _gated(hf, T=0)
    assert L.hobflops_gated_forward(ctypes.byref(empty), *[None] * 9, 0, None) == 0


def _w4(hf, x=FAKE, type=1, T=2, K=64, N=8, ldx=64, codes=FAKE, scales=FAKE, group=32, scale=1,
        y=FAKE, ldy=8):
    L = hf.lib()
    a = L.hobflops_w4_linear(x, type, T, K, N, ldx, codes, scales, group, scale, y, ldy, None)
    b = L.hobflops_w4_gated(x, type, T, K, N, ldx, codes, scales, codes, scales, group, scale, 0, y,
                            ldy, None)
    assert a == b
    return a


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), -1), (dict(K=0, ldx=0), -1), (dict(N=0, ldy=0), -1), (dict(ldx=63), -1),
    (dict(ldy=7), -1), (dict(type=0), -2), (dict(type=4), -1), (dict(group=48), -1),
    (dict(scale=4), -1), (dict(x=None), -1), (dict(codes=None), -1), (dict(scales=None), -1),
    (dict(y=None), -1), (dict(x=ODD), -3), (dict(y=ODD), -3), (dict(scales=ODD), -3)])
def test_w4_refusals(hf, bad, status):
    assert _w4(hf, **bad) == status


def test_w4_gated_activation(hf):
    L = hf.lib()
    for act in (-1, 3):
        assert L.hobflops_w4_gated(FAKE, 1, 2, 64, 8, 64, FAKE, FAKE, FAKE, FAKE, 32, 0, act, FAKE,
                                   8, None) == -1
    assert L.hobflops_w4_linear(None, 1, 0, 64, 8, 64, None, None, 32, 0, None, 8, None) == 0


def test_host_tensors_are_refused(hf):
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        hf.block_pack(x, (4, 3))
    with pytest.raises(TypeError):
        hf.gated_forward(x, x, x)
    with pytest.raises(TypeError):
        hf.w4_linear(x, x, x)


@pytest.mark.parametrize("f", [(4, 3), (5, 2), (2, 1)])
def test_reference_codes(f):
    """The reference's own rounding: every value is its code's, and every midpoint goes to the even
    code of its two."""
    v = ref.code_values(f)
    assert np.array_equal(ref.nearest_codes(v, f), np.arange(len(v)))
    mid = (v[1:] + v[:-1]) / 2
    assert (ref.nearest_codes(mid, f) % 2 == 0).all()
    assert v[-1] == {(4, 3): 448.0, (5, 2): 57344.0, (2, 1): 6.0}[f]
    for e in (-20, 0, 7):
        for m in (1.0, 1.5, 1.75, 1.8125, 1.81251, 1.875, 1.99):
            k = ref.pow2_scale(m * 2.0 ** e, f)
            n = m * 2.0 ** (e - k)
            assert n < v[-1] * 1.2 and 2 * n > v[-1]


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_reference_gradient_by_differences(kind):
    g = np.linspace(-6, 6, 481)[np.newaxis] + 0.0007
    h = 1e-5
    num = (ref.act(g + h, kind)[0] - ref.act(g - h, kind)[0]) / (2 * h)
    assert np.abs(num - ref.act(g, kind)[1]).max() < 1e-8
