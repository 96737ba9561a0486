"""The gated block on the GPU against a plain 64-bit reference.

Tolerances, derived: a float32 sum of n products is at most n 2^-23 sum |a b| off (each product's
and each addition's rounding, with a factor of two for the order), the activations at most 2^-19 of
their argument's size (exponential, division, erf), and an output's rounding to its type at most
half a step: u |y| with u = 2^-9 (bfloat16), 2^-12 (float16), plus float16's smallest step. The gradients
of g and u are rounded to the type once more before their products.
"""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # a whole step: twice the rounding
TINY = {"bf16": 0.0, "f16": 2.0 ** -24}
EPS, ACT = 2.0 ** -23, 2.0 ** -19


def _make(rows, cols, dtype, seed, scale=1.0, ld=None, offset=0):
    """Rows of a wider, possibly misaligned tensor: (GPU view, float64 array)."""
    ld = ld or cols
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, ld), generator=g) * scale).to(TYPES[dtype])
    flat = torch.zeros(rows * ld + offset, dtype=x.dtype)
    flat[offset:] = x.reshape(-1)
    view = flat.cuda()[offset:].view(rows, ld)[:, :cols]
    return view, view.double().cpu().numpy()


def _blocks(hf, saved, cols):
    """float64 values, and the scale factors, of a saved (codes, scales) in format f."""
    (codes, scales), f = saved
    factors = np.exp2(scales.cpu().double().numpy() - 127)
    return ref.unpack(codes.cpu().numpy().astype(np.int64), factors, f), factors


def _forward_bounds(x, wg, wu, act):
    D = x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = (D * EPS * (np.abs(x) @ np.abs(w).T) for w in (wg, wu))
    a = ref.act(g, act)[0]
    ea = 1.13 * eg + ACT * np.abs(g)
    return g, u, eg, eu, a * u, ea * (np.abs(u) + eu) + np.abs(a) * eu


def _check_blocks(q, factors, v, ev, f):
    """q: what the blocks of values within ev of v stand for. The scale is that of a value in
    that range, and every code one of the nearest to a value in that range."""
    top = ref.code_values(f)[-1]
    wF = f[1]
    low = 2.0 ** (1 - (2 ** (f[0] - 1) - 1) - wF)
    T, F = v.shape
    for g in range(factors.shape[1]):
        s = slice(32 * g, 32 * g + 32)
        lo, hi = (np.abs(v[:, s]) - ev[:, s]).max(1), (np.abs(v[:, s]) + ev[:, s]).max(1)
        for t in range(T):
            k0, k1 = ref.pow2_scale(max(lo[t], 0.0), f), ref.pow2_scale(hi[t], f)
            assert 2.0 ** k0 <= factors[t, g] <= 2.0 ** k1
    sc = np.repeat(factors, 32, 1)[:, :F]
    n = (np.abs(v) + ev) / sc
    step = np.exp2(np.floor(np.log2(np.maximum(n, low))) - wF)
    step = np.maximum(step, low)
    assert (np.abs(q - v) <= (step / 2 + (n > top) * step) * sc + ev).all()


SHAPES = [  # T, D, F, (ldx, ldw, ldh), offset of every tensor in elements
    (1, 1, 1, None, 0), (1, 64, 32, None, 0), (3, 40, 33, None, 0), (17, 72, 100, (80, 88, 104), 0),
    (5, 37, 31, None, 0), (64, 128, 128, None, 0), (65, 136, 260, None, 8), (129, 200, 70, None, 1),
    (16, 256, 512, None, 0), (300, 96, 257, (99, 97, 301), 3), (260, 520, 264, None, 0),
    (2, 1030, 96, None, 0), (40, 2048, 64, None, 0), (33, 64, 600, (64, 64, 602), 0)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:3])))
@pytest.mark.parametrize("dtype,act", [("bf16", 0), ("f16", 1), ("bf16", 2), ("f16", 0)])
def test_forward(shape, dtype, act):
    hf = need_gpu()
    T, D, F, lds, off = shape
    lds = lds or (D, D, F)
    say("forward", shape, dtype, act)
    xt, x = _make(T, D, dtype, 1, 1.0, lds[0], off)
    gt, wg = _make(F, D, dtype, 2, 2.0 / D ** 0.5, lds[1], off)
    ut, wu = _make(F, D, dtype, 3, 1.0 / D ** 0.5, lds[1], off)
    out = torch.full((T * lds[2] + off,), 7.0, dtype=TYPES[dtype], device="cuda")
    out = out[off:].view(T, lds[2])
    h = hf.gated_forward(xt, gt, ut, act, out=out[:, :F])
    assert h.data_ptr() == out.data_ptr()
    g, u, eg, eu, want, e = _forward_bounds(x, wg, wu, act)
    got = h.double().cpu().numpy()
    assert (np.abs(got - want) <= e + UNIT[dtype] * np.abs(want) + TINY[dtype]).all()
    assert (out[:, F:] == 7.0).all()
    f = (4, 3) if dtype == "bf16" else (5, 2)
    h2, saved = hf.gated_forward(xt, gt, ut, act, ckpt=f)
    assert torch.equal(h2, h)
    assert np.array_equal(_blocks(hf, (saved.x, f), D)[0], ref.unpack(*ref.pack(x, f), f))
    for s, v, ev in ((saved.gate, g, eg), (saved.up, u, eu)):
        _check_blocks(*_blocks(hf, (s, f), F), v, ev, f)


def _backward_case(hf, T, D, F, dtype, f, lds, off, act):
    xt, x = _make(T, D, dtype, 4)
    gt, wg = _make(F, D, dtype, 5, 2.0 / D ** 0.5, lds[1], off)
    ut, wu = _make(F, D, dtype, 6, 1.0 / D ** 0.5, lds[1], off)
    dt, dh = _make(T, F, dtype, 7, 0.25, lds[2], off)
    # the checkpoints are inputs: of the products' own values, the format's small and large ones too
    blocks = []
    for v, seed in ((x, 0), (x @ wg.T, 8), (x @ wu.T, 9)):
        t = torch.from_numpy(v).float()
        if seed:
            t = t * torch.exp2(torch.randint(-9, 3, t.shape,
                                             generator=torch.Generator().manual_seed(seed)).float())
        blocks.append(hf.block_pack(t.cuda(), f))
    saved = hf.GatedSaved(*blocks, hf.fmt(f))
    xq, gq, uq = (_blocks(hf, (b, f), 0)[0] for b in blocks)
    return (xt, gt, ut, dt), saved, (dh, wg, wu, xq, gq, uq)


def _gradients(dh, wg, wu, xq, gq, uq, dtype, act):
    """The formulas' gradients of x, w_gate and w_up, each with how far off it may be."""
    T, F = dh.shape
    a, da = ref.act(gq, act)
    dg, du = dh * uq * da, dh * a
    # off by the activation's error and the rounding to the type
    eg = np.abs(dh * uq) * ACT * (1 + np.abs(gq)) + UNIT[dtype] * np.abs(dg) + TINY[dtype]
    eu = np.abs(dh) * ACT * np.abs(gq) + UNIT[dtype] * np.abs(du) + TINY[dtype]
    ag, au = np.abs(dg) + eg, np.abs(du) + eu
    for want, e in (
            (dg @ wg + du @ wu,
             eg @ np.abs(wg) + eu @ np.abs(wu) + 2 * F * EPS * (ag @ np.abs(wg) + au @ np.abs(wu))),
            (dg.T @ xq, eg.T @ np.abs(xq) + T * EPS * (ag.T @ np.abs(xq))),
            (du.T @ xq, eu.T @ np.abs(xq) + T * EPS * (au.T @ np.abs(xq)))):
        yield want, e * (1 + UNIT[dtype]) + UNIT[dtype] * np.abs(want) + TINY[dtype]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:3])))
@pytest.mark.parametrize("dtype,f,act", [("bf16", (4, 3), 0), ("f16", (5, 2), 1),
                                         ("bf16", (5, 2), 2), ("f16", (4, 3), 0)])
def test_backward(shape, dtype, f, act):
    hf = need_gpu()
    T, D, F, lds, off = shape
    lds = lds or (D, D, F)
    say("backward", shape, dtype, f, act)
    (xt, gt, ut, dt), saved, (dh, wg, wu, xq, gq, uq) = _backward_case(hf, T, D, F, dtype, f, lds,
                                                                      off, act)
    dx, dwg, dwu = hf.gated_backward(dt, saved, gt, ut, act)
    for got, (want, bound) in zip((dx, dwg, dwu), _gradients(dh, wg, wu, xq, gq, uq, dtype, act)):
        got = got.double().cpu().numpy()
        assert got.shape == want.shape
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / (bound + 1e-300)).max())
    again = hf.gated_backward(dt, saved, gt, ut, act)
    assert all(torch.equal(p, q) for p, q in zip((dx, dwg, dwu), again))


@pytest.mark.parametrize("act", [0, 1])
def test_gradients_by_differences(act):
    """The gradients against central differences of L = sum(dh * act(g) * u) in 64 bits at the
    checkpoints' values, along random directions of x, w_gate and w_up."""
    hf = need_gpu()
    T, D, F = 24, 40, 56
    (xt, gt, ut, dt), saved, (dh, wg, wu, xq, gq, uq) = _backward_case(hf, T, D, F, "bf16", (4, 3),
                                                                      (D, D, F), 0, act)
    dx, dwg, dwu = (t.double().cpu().numpy() for t in hf.gated_backward(dt, saved, gt, ut, act))

    def loss(x=0.0, vg=0.0, vu=0.0):
        g = gq + x * np.ones((T, D)) @ wg.T + xq @ (vg * np.ones((F, D))).T
        u = uq + x * np.ones((T, D)) @ wu.T + xq @ (vu * np.ones((F, D))).T
        return float((dh * ref.act(g, act)[0] * u).sum())

    rng = np.random.default_rng(3)
    h = 1e-5
    bounds = [b for _, b in _gradients(dh, wg, wu, xq, gq, uq, "bf16", act)]
    for name, got, bound in (("x", dx, bounds[0]), ("vg", dwg, bounds[1]), ("vu", dwu, bounds[2])):
        for _ in range(3):
            v = rng.standard_normal(got.shape)
            num = (loss(**{name: h * v}) - loss(**{name: -h * v})) / (2 * h)
            # the difference's own error: h^2 times a third derivative, and rounding over h
            assert abs(num - (got * v).sum()) <= (bound * np.abs(v)).sum() + 1e-5 * (1 + abs(num))


def test_no_tokens():
    hf = need_gpu()
    w = torch.ones(40, 24, dtype=torch.bfloat16, device="cuda")
    h, saved = hf.gated_forward(w[:0], w, w, ckpt=(4, 3))
    assert h.shape == (0, 40)
    dx, dwg, dwu = hf.gated_backward(h, saved, w, w)
    assert dx.shape == (0, 24) and not dwg.any() and not dwu.any() and dwg.shape == (40, 24)


@pytest.mark.parametrize("D", [64, 61])
def test_what_is_not_finite_stays_where_it_belongs(D):
    """A NaN or infinity in one token reaches that token's outputs alone, one in a row of a weight that
    row's column alone, also where rows end inside a tile and the row after holds them."""
    hf = need_gpu()
    T, F = 37, 45
    xt, x = _make(T, D, "bf16", 11)
    gt, _ = _make(F, D, "bf16", 12, D ** -0.5)
    ut, _ = _make(F, D, "bf16", 13, D ** -0.5)
    base, saved0 = hf.gated_forward(xt, gt, ut, ckpt=(4, 3))
    xt, gt = xt.clone(), gt.clone()
    xt[7, 0], xt[20, D - 1] = float("nan"), float("inf")
    gt[33, 0] = float("nan")
    h, saved = hf.gated_forward(xt, gt, ut, ckpt=(4, 3))
    clean = torch.ones(T, F, dtype=torch.bool)
    clean[[7, 20]] = False
    clean[:, 33] = False
    assert torch.equal(h.cpu()[clean], base.cpu()[clean])
    assert h[7].isnan().all() and h[:, 33].isnan().all() and not h[20].isfinite().any()
    g0, g1 = (hf.block_unpack(*s.gate, F, (4, 3)).cpu() for s in (saved0, saved))
    assert torch.equal(g0[clean], g1[clean])
    dt, _ = _make(T, F, "bf16", 14)
    dx0, dg0, du0 = hf.gated_backward(dt, saved0, gt.nan_to_num(), ut)
    dt = dt.clone()
    dt[5, 3] = float("nan")
    dx, dg, du = hf.gated_backward(dt, saved0, gt.nan_to_num(), ut)
    rows = torch.arange(T) != 5
    cols = torch.arange(F) != 3
    assert torch.equal(dx.cpu()[rows], dx0.cpu()[rows]) and dx[5].isnan().all()
    for a, b in ((dg, dg0), (du, du0)):
        assert torch.equal(a.cpu()[cols], b.cpu()[cols]) and a[3].isnan().all()


def test_streams_and_repeats():
    """On a stream of its own, interleaved with calls of other sizes: the same bits."""
    hf = need_gpu()
    sizes = [(70, 136, 264), (5, 72, 96), (200, 64, 128)]
    data = [[_make(a, b, "bf16", i, 0.3)[0] for i, (a, b) in enumerate(
        ((T, D), (F, D), (F, D), (T, F)))] for T, D, F in sizes]

    def step(x, wg, wu, dh):
        h, saved = hf.gated_forward(x, wg, wu, ckpt=(4, 3))
        return (h,) + hf.gated_backward(dh, saved, wg, wu)

    first = [step(*d) for d in data]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        second = [[step(*d) for d in data] for _ in range(3)]
    s.synchronize()
    for rep in second:
        for a, b in zip(first, rep):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_graph():
    """Forward and backward in a HIP graph, replayed with new inputs between eager calls."""
    hf = need_gpu()
    T, D, F = 70, 136, 264
    x, wg, wu, dh = (_make(a, b, "bf16", i, 0.3)[0].clone() for i, (a, b) in enumerate(
        ((T, D), (F, D), (F, D), (T, F))))

    def step():
        h, saved = hf.gated_forward(x, wg, wu, ckpt=(4, 3))
        return (h,) + hf.gated_backward(dh, saved, wg, wu)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        x.copy_(_make(T, D, "bf16", 50 + i, 0.3)[0])
        graph.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, step()))


def _act64(g, act):
    if act == 0:
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if act == 1:
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g * g / 2) / (2 * np.pi) ** 0.5
    return g.clamp(min=0), (g > 0).double()


def _within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert not off.isnan().any() and off.max() <= 0, (what, float(off.max()))


@pytest.mark.parametrize("T,D,F,dtype,f,act", [
    (520, 136, 12500, "bf16", (4, 3), 0),      # ragged large tiles of the forward product
    (4000, 2056, 2800, "f16", (5, 2), 1),      # and of both gradients
    (4096, 2048, 3008, "bf16", (4, 3), 0),
    (700, 264, 3000, "bf16", (5, 2), 2),       # small tiles, many of them
    (30, 1000, 9000, "f16", (4, 3), 0),        # a long sum in parts
    (2500, 4096, 40, "bf16", (4, 3), 1)])
def test_large(T, D, F, dtype, f, act):
    """The kernels of large sizes, with the bounds above, against torch in 64 bits on the GPU."""
    hf = need_gpu()
    say("large", T, D, F, dtype, f, act)
    (xt, _), (gt, _), (ut, _), (dt, _) = (
        _make(r, c, dtype, 20 + i, s) for i, (r, c, s) in enumerate(
            ((T, D, 1.0), (F, D, 2.0 / D ** 0.5), (F, D, 1.0 / D ** 0.5), (T, F, 0.25))))
    x, wg, wu, dh = (t.double() for t in (xt, gt, ut, dt))
    h, saved = hf.gated_forward(xt, gt, ut, act, ckpt=f)
    g, u = x @ wg.T, x @ wu.T
    eg, eu = (D * EPS * (x.abs() @ w.abs().T) for w in (wg, wu))
    a = _act64(g, act)[0]
    _within(h, a * u, (1.13 * eg + ACT * g.abs()) * (u.abs() + eu) + a.abs() * eu +
            UNIT[dtype] * (a * u).abs() + TINY[dtype], "h")
    assert torch.equal(hf.gated_forward(xt, gt, ut, act), h)
    q = [hf.block_unpack(*b, c, f).double() for b, c in ((saved.x, D), (saved.gate, F), (saved.up, F))]
    for v, ev, b, name in ((g, eg, q[1], "gate"), (u, eu, q[2], "up")):
        # a scale at most twice what the group's largest value needs: half a step of that binade
        pad = torch.nn.functional.pad(v.abs() + ev, (0, -F % 32)).reshape(T, -1, 32)
        low = 2.0 ** (1 - f[1] - (2 ** (f[0] - 1) - 1) - (8 if f == (4, 3) else 15))
        small = (pad.amax(2) * 2 * low).repeat_interleave(32, 1)[:, :F]
        _within(b, v, ev + (v.abs() + ev) * 2.0 ** -f[1] / 2 + small, name)
    xq, gq, uq = q
    a, da = _act64(gq, act)
    dg, du = dh * uq * da, dh * a
    eg = (dh * uq).abs() * ACT * (1 + gq.abs()) + UNIT[dtype] * dg.abs() + TINY[dtype]
    eu = dh.abs() * ACT * gq.abs() + UNIT[dtype] * du.abs() + TINY[dtype]
    ag, au = dg.abs() + eg, du.abs() + eu
    grads = hf.gated_backward(dt, saved, gt, ut, act)
    for got, want, e, name in (
            (grads[0], dg @ wg + du @ wu, eg @ wg.abs() + eu @ wu.abs() +
             2 * F * EPS * (ag @ wg.abs() + au @ wu.abs()), "dx"),
            (grads[1], dg.T @ xq, eg.T @ xq.abs() + T * EPS * (ag.T @ xq.abs()), "dw_gate"),
            (grads[2], du.T @ xq, eu.T @ xq.abs() + T * EPS * (au.T @ xq.abs()), "dw_up")):
        _within(got, want, e * (1 + UNIT[dtype]) + UNIT[dtype] * want.abs() + TINY[dtype], name)
    again = hf.gated_backward(dt, saved, gt, ut, act)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))
