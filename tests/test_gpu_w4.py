"""Products with 4-bit weights on the GPU against a plain 64-bit reference.

Tolerance, derived: K products summed in float32 in some order, the scale applied to parts of the
sum: (K + 4) 2^-23 sum |x w|, and the output's rounding; of the gated form the errors of both
products through the activation (slope at most 1.13, its own error 2^-19 of its argument).
"""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 0.0, "f16": 2.0 ** -24}
EPS, ACT = 2.0 ** -23, 2.0 ** -19
SCALES = {"pow2": 0, "bf16": 1, "f32": 2}


def _weights(hf, N, K, group, scale, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((N, K), generator=g) * K ** -0.5
    codes, scales = hf.block_pack(w.cuda(), (2, 1), group=group, scale=SCALES[scale])
    f = scales.cpu().double().numpy()
    f = np.exp2(f - 127) if scale == "pow2" else f
    return codes, scales, ref.unpack(ref.nibbles(codes.cpu().numpy(), K), f, (2, 1), group)


def _x(T, K, dtype, seed, ld=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    ld = ld or K
    flat = torch.randn(T * ld + offset, generator=g).to(TYPES[dtype]).cuda()
    return flat[offset:].view(T, ld)[:, :K]


SHAPES = [(1, 1, 1), (1, 32, 16), (1, 33, 5), (2, 64, 7), (3, 130, 33), (1, 4096, 40), (1, 2056, 17),
          (4, 256, 64), (5, 1000, 50), (8, 512, 129), (9, 520, 31), (16, 1024, 48), (17, 264, 100),
          (33, 136, 65), (64, 2080, 20), (100, 72, 30), (1, 31, 3), (7, 8200, 9)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,group,scale", [("bf16", 32, "pow2"), ("f16", 64, "bf16"),
                                               ("bf16", 128, "f32"), ("f16", 32, "f32"),
                                               ("bf16", 128, "bf16")])
def test_linear_and_gated(shape, dtype, group, scale):
    hf = need_gpu()
    T, K, N = shape
    say("w4", shape, dtype, group, scale)
    cg, sg, wg = _weights(hf, N, K, group, scale, 1)
    cu, su, wu = _weights(hf, N, K, group, scale, 2)
    for ld, off in ((None, 0), (K + 3, 1)):
        xt = _x(T, K, dtype, 3, ld, off)
        x = xt.double().cpu().numpy()
        g, u = x @ wg.T, x @ wu.T
        eg, eu = ((K + 4) * EPS * (np.abs(x) @ np.abs(w).T) for w in (wg, wu))
        out = torch.full((T, N + 2), 7.0, dtype=TYPES[dtype], device="cuda")
        y = hf.w4_linear(xt, cg, sg, group=group, out=out[:, :N]).double().cpu().numpy()
        assert (np.abs(y - g) <= eg + UNIT[dtype] * np.abs(g) + TINY[dtype]).all()
        assert (out[:, N:] == 7.0).all()
        for act in (0, 1, 2):
            h = hf.w4_gated(xt, cg, sg, cu, su, act, group=group).double().cpu().numpy()
            a = ref.act(g, act)[0]
            e = (1.13 * eg + ACT * np.abs(g)) * (np.abs(u) + eu) + np.abs(a) * eu
            want = a * u
            assert (np.abs(h - want) <= e + UNIT[dtype] * np.abs(want) + TINY[dtype]).all()


@pytest.mark.parametrize("T", [1, 3, 6, 20])
@pytest.mark.parametrize("group,scale", [(32, "pow2"), (64, "f32")])
def test_all_codes_exactly(T, group, scale):
    """x with one 1 a token picks single weights: every code of every place, exactly."""
    hf = need_gpu()
    K, N = 160, 24
    rng = np.random.default_rng(4)
    packed = torch.from_numpy(rng.integers(0, 256, (N, K // 2), dtype=np.uint8)).cuda()
    groups = -(-K // group)
    if scale == "pow2":
        scales = torch.from_numpy(rng.integers(117, 131, (N, groups), dtype=np.uint8)).cuda()
        f = np.exp2(scales.cpu().double().numpy() - 127)
    else:
        scales = torch.exp2(torch.randint(-9, 4, (N, groups)).float()).cuda()
        f = scales.cpu().double().numpy()
    w = ref.unpack(ref.nibbles(packed.cpu().numpy(), K), f, (2, 1), group)
    for k0 in range(0, K, T):
        n = min(T, K - k0)
        x = torch.zeros(T, K, dtype=torch.bfloat16)
        x[torch.arange(n), k0 + torch.arange(n)] = 1.0
        y = hf.w4_linear(x.cuda(), packed, scales, group=group).double().cpu().numpy()
        assert np.array_equal(y[:n], w[:, k0:k0 + n].T) and not y[n:].any()


@pytest.mark.parametrize("T", [1, 2, 5, 18])
def test_what_is_not_finite(T):
    """An infinity or NaN of a token reaches that token's outputs alone; a NaN scale its row's."""
    hf = need_gpu()
    K, N = 200, 37
    codes, scales, w = _weights(hf, N, K, 32, "pow2", 5)
    x = _x(T, K, "bf16", 6).clone()
    base = hf.w4_linear(x, codes, scales).clone()
    x[T - 1, 0] = float("inf")
    scales = scales.clone()
    scales[11, 2] = 255
    y = hf.w4_linear(x, codes, scales)
    rows = torch.arange(N) != 11
    assert torch.equal(y[:T - 1].cpu()[:, rows], base[:T - 1].cpu()[:, rows])
    assert y[:, 11].isnan().all()
    last = y[T - 1].cpu()[rows].double().numpy()
    w0 = w[rows.numpy(), 0]
    assert np.isnan(last[w0 == 0]).all()
    assert np.array_equal(last[w0 != 0], np.sign(w0[w0 != 0]) * np.inf)


def test_no_tokens_and_streams():
    hf = need_gpu()
    codes, scales, w = _weights(hf, 40, 64, 32, "pow2", 7)
    assert hf.w4_linear(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), codes,
                        scales).shape == (0, 40)
    x = _x(3, 64, "bf16", 8)
    y = hf.w4_linear(x, codes, scales)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        z = [hf.w4_linear(x, codes, scales) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(y, t) for t in z)


def test_arguments():
    hf = need_gpu()
    codes, scales, _ = _weights(hf, 40, 64, 32, "pow2", 7)
    x = _x(3, 64, "bf16", 8)
    with pytest.raises(ValueError):
        hf.w4_linear(x, codes, scales, group=48)
    with pytest.raises(ValueError):
        hf.w4_linear(x, codes, scales[:, :1].contiguous())
    with pytest.raises(ValueError):
        hf.w4_linear(x[:, ::2], codes, scales)
    with pytest.raises(hf.HobflopsError):
        hf.w4_linear(x.float(), codes, scales)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,N,K", [(1, 260, 256), (3, 300, 96), (20, 257, 256), (16, 256, 16640)])
def test_every_power_of_two(dtype, T, N, K):
    """Scale bytes from 0 to 255, one a row, mixed within a row and alone: weights picked one by one are
    the code's value times the scale, rounded to the type once."""
    hf = need_gpu()
    rng = np.random.default_rng(9)
    packed = torch.from_numpy(rng.integers(0, 256, (N, K // 2), dtype=np.uint8)).cuda()
    groups = K // 32
    b = np.repeat((np.arange(N) % 256)[:, None], groups, 1)
    b[:, 1::3] = 127                 # ordinary scales between them
    b[200:] = np.minimum(b[200:], 254)
    scales = torch.from_numpy(b.astype(np.uint8)).cuda()
    f = np.where(b == 255, np.nan, np.exp2(b - 127.0))
    codes = ref.nibbles(packed.cpu().numpy(), K)
    with np.errstate(invalid="ignore", over="ignore"):
        w = ref.unpack(codes, f, (2, 1)).astype(np.float32)
    for k0 in list(range(0, min(K, 256) - T, max(T, 16))) + [K - T]:
        x = torch.zeros(T, K, dtype=TYPES[dtype])
        x[torch.arange(T), k0 + torch.arange(T)] = 1.0
        y = hf.w4_linear(x.cuda(), packed, scales).cpu()
        want = torch.from_numpy(w[:, k0:k0 + T].T.copy()).to(TYPES[dtype])
        nan = torch.from_numpy(np.isnan(f).any(1))  # a NaN scale is its whole row's
        assert y[:, nan].isnan().all()
        assert torch.equal(y[:, ~nan], want[:, ~nan])


@pytest.mark.parametrize("T,K,N,group,scale", [
    (1, 4096, 11300, 32, "pow2"), (5, 4104, 9001, 64, "f32"), (16, 1280, 20000, 128, "bf16"),
    (2, 8192, 5000, 32, "f32"), (16, 11264, 600, 32, "pow2"), (40, 2048, 1500, 64, "bf16"),
    (40, 2048, 8300, 64, "bf16"), (70, 264, 9001, 32, "pow2"), (64, 1096, 8192, 128, "f32"),
    (17, 136, 8185, 32, "f32"), (130, 4096, 4104, 32, "pow2")])
def test_many_tiles(T, K, N, group, scale):
    """Sizes at which a workgroup takes several tiles, or a wave several rounds."""
    hf = need_gpu()
    say("w4 many tiles", T, K, N, group, scale)
    for dtype in TYPES:
        cg, sg, wg = _weights(hf, N, K, group, scale, 11)
        cu, su, wu = _weights(hf, N, K, group, scale, 12)
        xt = _x(T, K, dtype, 13)
        x = xt.double()
        wg, wu = torch.from_numpy(wg).cuda(), torch.from_numpy(wu).cuda()
        g, u = x @ wg.T, x @ wu.T
        eg, eu = ((K + 4) * EPS * (x.abs() @ w.abs().T) for w in (wg, wu))
        y = hf.w4_linear(xt, cg, sg, group=group).double()
        assert ((y - g).abs() <= eg + UNIT[dtype] * g.abs() + TINY[dtype]).all()
        s = torch.sigmoid(g)
        h = hf.w4_gated(xt, cg, sg, cu, su, 0, group=group).double()
        e = (1.13 * eg + ACT * g.abs()) * (u.abs() + eu) + (g * s).abs() * eu
        want = g * s * u
        assert ((h - want).abs() <= e + UNIT[dtype] * want.abs() + TINY[dtype]).all()
        assert torch.equal(hf.w4_linear(xt, cg, sg, group=group).double(), y)


@pytest.mark.parametrize("T,ld", [(3, (1 << 26) - 2), (16, (1 << 25) + 2), (40, (1 << 25) + 2), (40, 1 << 24)])
def test_rows_far_apart(T, ld):
    """Rows of x and y whose offsets pass 31 bits, K that ends inside a step."""
    hf = need_gpu()
    say("w4 rows far apart", T, ld)
    K, N, group = 136, 8200, 32
    cg, sg, wg = _weights(hf, N, K, group, "f32", 21)
    near = _x(T, K, "bf16", 22)
    x = torch.full((T * ld,), float("nan"), dtype=torch.bfloat16, device="cuda").view(T, ld)[:, :K]
    x.copy_(near)
    out = torch.empty((T * ld,), dtype=torch.bfloat16, device="cuda").view(T, ld)[:, :N]
    y = hf.w4_linear(x, cg, sg, group=group, out=out).double()
    wg = torch.from_numpy(wg).cuda()
    want = near.double() @ wg.T
    e = (K + 4) * EPS * (near.double().abs() @ wg.abs().T)
    assert ((y - want).abs() <= e + UNIT["bf16"] * want.abs()).all()
