"""The AdamW step on the GPU: every output equals float32 operations rounded one by one, bit for bit."""
import numpy as np
import pytest
import torch

import narrow_ref
import step_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F = np.float32


def _flat(arrays):
    """Arrays one after the other, each filled up with zeros to a multiple of 32."""
    return np.concatenate([np.pad(a, (0, -len(a) % 32)) for a in arrays] or [np.zeros(0, F)])


def _parts(flat, sizes):
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + n])
        at += -(-n // 32) * 32
    return out


def _state_np(hf, state):
    f = state.fmt
    if f is None:
        return state.m.cpu().numpy().copy(), state.v.cpu().numpy().copy()
    m, r = (ref.decode(c.cpu().numpy(), s.cpu().numpy(), f) for c, s in (state.m, state.v))
    return m, r * r


def _same_codes(got, want, f):
    """A NaN has any sign: which one an invalid operation gives differs between machines."""
    got, want, low = got.astype(np.int64), want.copy(), 2 ** sum(f) - 1
    for c in (got, want):
        c[np.isnan(narrow_ref.decode(c, f))] = low
    return np.array_equal(got, want)


def _grads(rng, sizes, spread=6.0):
    return [(rng.standard_normal(n) * np.exp2(rng.uniform(-spread, spread, n)) * 1e-3).astype(F) for n in sizes]


def _run(hf, sizes, gtype, fmt, ctype, steps=3, offset=0, seed=99, scale=1.0, first=1, **kw):
    rng = np.random.default_rng(5)
    start = [rng.standard_normal(n).astype(F) for n in sizes]
    params = [torch.empty(n + offset, device="cuda")[offset:].copy_(torch.from_numpy(p))
              for n, p in zip(sizes, start)]
    copies = [torch.empty(n + offset, dtype=TYPES[ctype], device="cuda")[offset:] for n in sizes] if ctype else None
    state = hf.adamw_state(params, fmt)
    assert hf.adamw_places(params)[1] == sum(-(-n // 32) * 32 for n in sizes)
    args = dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, **kw)
    p = _flat(start)
    for step in range(first, first + steps):
        g = [t.to(TYPES[gtype]) for t in map(torch.from_numpy, _grads(rng, sizes))]
        m, v = _state_np(hf, state)
        dev = [torch.empty(n + offset, dtype=TYPES[gtype], device="cuda")[offset:].copy_(t) for n, t in zip(sizes, g)]
        hf.adamw(params, dev, state, step, copies=copies, grad_scale=scale, seed=seed, **args)
        p, m, v, r = ref.adamw(p, _flat([t.float().numpy() for t in g]), m, v, step, args["lr"], args["betas"],
                               args["eps"], args["weight_decay"], scale)
        for got, want in zip(params, _parts(p, sizes)):
            assert np.array_equal(got.cpu().numpy(), want)
        if copies:
            for got, want in zip(copies, _parts(p, sizes)):
                assert torch.equal(got.cpu(), torch.from_numpy(want.copy()).to(TYPES[ctype]))
        if fmt is None:
            for got, want in ((state.m, m), (state.v, v)):
                assert np.array_equal(got.cpu().numpy(), want)
        else:
            um, ur = ref.uniform(np.arange(len(m)), step, seed)
            for (codes, scales), x, u, sq in ((state.m, m, um, None), (state.v, r, ur, v)):
                want, k, _ = ref.encode(x, u, fmt, sq)
                assert np.array_equal(scales.cpu().numpy().astype(int), k + 127)
                assert _same_codes(codes.cpu().numpy(), want, fmt)
    return params, state


SIZES = [[1], [7], [32], [33, 1, 64], [4096], [2048, 2049, 5], [100000], [31] * 70, [1 + 97 * (i * i % 41) for i in range(130)]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("gtype,fmt,ctype", [("f32", None, None), ("bf16", None, "bf16"), ("f16", (4, 3), "f16"),
                                             ("f32", (5, 2), None), ("bf16", (4, 3), "bf16"), ("f16", (5, 2), None)])
def test_steps(sizes, gtype, fmt, ctype):
    hf = need_gpu()
    say("adamw", len(sizes), max(sizes), gtype, fmt, ctype)
    _run(hf, sizes, gtype, fmt, ctype)


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("fmt", [None, (4, 3)])
def test_misaligned(offset, fmt):
    hf = need_gpu()
    _run(hf, [5000, 33], "f16", fmt, "bf16", offset=offset)


@pytest.mark.parametrize("fmt", [None, (5, 2)])
def test_large(fmt):
    """More values than one round of a workgroup."""
    hf = need_gpu()
    _run(hf, [(1 << 22) + 77, 3, 70001], "bf16", fmt, "bf16", steps=2)


def test_a_scale_and_a_late_step():
    hf = need_gpu()
    _run(hf, [333], "f16", (4, 3), None, scale=1 / 1024, first=100000, seed=(1 << 60) + 5)
    _run(hf, [333], "f16", None, None, scale=1 / 1024, first=1 << 33)


def test_some_tensors_have_no_gradient():
    hf = need_gpu()
    sizes = [40, 50, 60]
    rng = np.random.default_rng(6)
    params = [torch.from_numpy(rng.standard_normal(n).astype(F)).cuda() for n in sizes]
    grads = [torch.from_numpy(g).cuda() for g in _grads(rng, sizes)]
    full = [p.clone() for p in params]
    a, b = hf.adamw_state(params, (4, 3)), hf.adamw_state(params, (4, 3))
    before = params[1].clone()
    hf.adamw(params, [grads[0], None, grads[2]], a, 1)
    hf.adamw(full, grads, b, 1)
    assert torch.equal(params[1], before) and torch.equal(params[0], full[0]) and torch.equal(params[2], full[2])
    assert (a.m[0][64:128] == 0).all() and torch.equal(a.m[0][128:], b.m[0][128:])
    hf.adamw(params, [None] * 3, a, 2)
    hf.adamw([], [], a, 2)
    copies = [None, torch.empty(50, dtype=torch.bfloat16, device="cuda"), None]
    hf.adamw(full, grads, b, 2, copies=copies)
    assert torch.equal(copies[1], full[1].bfloat16())


def test_values_on_the_device():
    """lr, step and grad_scale as tensors: the factors are those of the numbers, to the last place or the next."""
    hf = need_gpu()
    rng = np.random.default_rng(7)
    p0 = torch.from_numpy(rng.standard_normal(5000).astype(F)).cuda()
    g = torch.from_numpy(_grads(rng, [5000])[0]).cuda()
    for fmt in (None, (4, 3)):
        for step in (1, 2, 1000, 1 << 33):
            lr = float(F(1e-2))
            p, q = p0.clone(), p0.clone()
            a, b = hf.adamw_state([p], fmt), hf.adamw_state([q], fmt)
            hf.adamw([p], [g], a, step, lr=lr, grad_scale=0.5, seed=3)
            hf.adamw([q], [g], b, torch.tensor([step], device="cuda"), lr=torch.tensor(lr, device="cuda"),
                     grad_scale=torch.tensor(0.5, device="cuda"), seed=3)
            assert torch.allclose(p, q, rtol=2.0 ** -22, atol=lr * 2.0 ** -21)
            for s, t in ((a.m, b.m), (a.v, b.v)):
                for x, y in zip(*((s, t) if fmt else ((s,), (t,)))):
                    assert torch.equal(x, y)


@pytest.mark.parametrize("fmt", [None, (4, 3)])
def test_a_step_that_is_skipped(fmt):
    hf = need_gpu()
    p = torch.ones(100, device="cuda")
    g = torch.full((100,), float("inf"), device="cuda")
    s = hf.adamw_state([p], fmt)
    for value in (1.0, float("nan"), -2.0):
        hf.adamw([p], [g], s, 1, skip=torch.tensor([value], device="cuda"))
    assert (p == 1).all() and all((t == 0).all() for t in ([s.m, s.v] if fmt is None else [*s.m, *s.v]))
    hf.adamw([p], [torch.ones_like(p)], s, 1, skip=torch.zeros(1, device="cuda"))
    assert (p < 1).all()


@pytest.mark.parametrize("fmt", [None, (4, 3), (5, 2)])
def test_what_is_not_finite(fmt):
    """A gradient that is not finite spoils its own value alone; its group's others keep their scale."""
    hf = need_gpu()
    rng = np.random.default_rng(8)
    g = _grads(rng, [96])[0]
    p0 = rng.standard_normal(96).astype(F)
    results = []
    for bad in (False, True):
        h = g.copy()
        if bad:
            h[5], h[40], h[41] = np.nan, np.inf, -np.inf
        else:
            h[[5, 40, 41]] = 0
        p = torch.from_numpy(p0).cuda()
        s = hf.adamw_state([p], fmt)
        hf.adamw([p], [torch.from_numpy(h).cuda()], s, 1, seed=4)
        results.append([p] + ([s.m, s.v] if fmt is None else [s.m[0], s.v[0], s.m[1], s.v[1]]))
        if bad and fmt:
            m = narrow_ref.decode(s.m[0].cpu().numpy(), fmt)
            r = narrow_ref.decode(s.v[0].cpu().numpy(), fmt)
            assert np.isnan(m[5]) and np.isnan(r[5])
            assert (np.isnan(m[[40, 41]]).all() and np.isnan(r[[40, 41]]).all()) if fmt == (4, 3) else \
                (m[40] == np.inf and m[41] == -np.inf and (r[[40, 41]] == np.inf).all())
    ok = torch.ones(96, dtype=torch.bool, device="cuda")
    ok[[5, 40, 41]] = False
    for a, b in zip(*results):
        assert torch.equal(a[ok], b[ok]) if len(a) == 96 else torch.equal(a, b)
    assert results[1][0][~ok].isnan().all()


@pytest.mark.parametrize("fmt", [(4, 3), (5, 2)])
def test_small_and_large_moments(fmt):
    """Groups whose largest values lie anywhere in float32, zeros among them."""
    hf = need_gpu()
    rng = np.random.default_rng(9)
    n = 32 * 256
    g = (rng.standard_normal(n) * np.exp2(np.repeat(np.linspace(-149, 63, 256), 32))).astype(F)
    g[rng.random(n) < 0.2] = 0
    p = torch.zeros(n, device="cuda")
    s = hf.adamw_state([p], fmt)
    m, v = np.zeros(n, F), np.zeros(n, F)
    for step in (1, 2):
        hf.adamw([p], [torch.from_numpy(g).cuda()], s, step, seed=1, betas=(0.5, 0.75))
        _, m, v, r = ref.adamw(np.zeros(n, F), g, m, v, step, 1e-3, (0.5, 0.75), 1e-8, 0.01)
        um, ur = ref.uniform(np.arange(n), step, 1)
        for (codes, scales), x, u, sq in ((s.m, m, um, None), (s.v, r, ur, v)):
            want, k, _ = ref.encode(x, u, fmt, sq)
            assert _same_codes(codes.cpu().numpy(), want, fmt)
            assert np.array_equal(scales.cpu().numpy().astype(int), k + 127)
        m, v = _state_np(hf, s)


def test_what_a_state_is_can_be_read_as_blocks():
    hf = need_gpu()
    params, state = _run(hf, [320, 64], "f32", (4, 3), None, steps=2)
    for codes, scales in (state.m, state.v):
        n = codes.numel()
        v = hf.block_unpack(codes.view(1, n), scales.view(1, n // 32), n, (4, 3))[0].cpu().numpy()
        assert np.array_equal(v, ref.decode(codes.cpu().numpy(), scales.cpu().numpy(), (4, 3)))


def test_autograd_sees_the_change():
    """A backward pass that needs the weights before a step is an error after it."""
    hf = need_gpu()
    p = torch.ones(8, device="cuda", requires_grad=True)
    loss = (p * p).sum()
    hf.adamw([p], [torch.ones(8, device="cuda")], hf.adamw_state([p]), 1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_arguments():
    hf = need_gpu()
    p, q = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    g = torch.ones(64, device="cuda")
    s = hf.adamw_state([p, q])
    ok = lambda **k: hf.adamw([p, q], [g, g], s, 1, **k)  # noqa: E731
    ok()
    before = p.clone()
    for bad in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0)):
        with pytest.raises(hf.HobflopsError):
            ok(**bad)
    with pytest.raises(hf.HobflopsError):
        hf.adamw([p, q], [g, g], s, 0)
    with pytest.raises(hf.HobflopsError):          # the same tensor twice
        hf.adamw([p, p], [g, g], s, 1)
    with pytest.raises(hf.HobflopsError):          # overlapping ones
        both = torch.ones(96, device="cuda")
        hf.adamw([both[:64], both[32:]], [g, g], s, 1)
    with pytest.raises(hf.HobflopsError):          # a gradient that is a weight
        hf.adamw([p, q], [q, g], s, 1)
    with pytest.raises(ValueError):
        hf.adamw([p], [g, g], s, 1)
    with pytest.raises(ValueError):
        hf.adamw([p, q], [g, g[:32]], s, 1)
    with pytest.raises(ValueError):
        hf.adamw([p, q[:32]], [g, g[:32]], hf.adamw_state([p, p]), 1)
    with pytest.raises(TypeError):
        hf.adamw([p, q], [g, g.half()], s, 1)
    with pytest.raises(TypeError):
        hf.adamw([p, q.double()], [g, g], s, 1)
    with pytest.raises(TypeError):
        hf.adamw([p, q], [g, g.cpu()], s, 1)
    with pytest.raises(TypeError):
        ok(copies=[p.clone(), None])
    with pytest.raises(ValueError):
        ok(copies=[p.half()])
    with pytest.raises(TypeError):
        ok(skip=1.0)
    with pytest.raises(TypeError):
        ok(lr=torch.ones(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        hf.adamw([p.view(8, 8).t()], [g.view(8, 8).t()], hf.adamw_state([p]), 1)
    assert torch.equal(p, before)
