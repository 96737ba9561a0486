"""What is not finite stays where it belongs in the kernels of large sizes: tiles of 256 x 256 of the gated
block's products, tiles of 64 tokens of the products with 4-bit weights."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say
from test_gpu_gated import _make
from test_gpu_w4 import EPS, TINY, TYPES, UNIT, _weights, _x

pytestmark = pytest.mark.gpu


def _same(a, b, rows=None, cols=None):
    """Equal but for these rows and columns, in which b has no finite value."""
    keep = torch.ones(a.shape, dtype=torch.bool, device=a.device)
    for r in rows or ():
        assert not b[r].isfinite().any()
        keep[r] = False
    for c in cols or ():
        assert not b[:, c].isfinite().any()
        keep[:, c] = False
    assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("T,D,F", [(4001, 2060, 2810), (4000, 2056, 2816), (520, 136, 10300)])
def test_gated(T, D, F):
    hf = need_gpu()
    say("isolation, gated", T, D, F)
    (x, _), (wg, _), (wu, _), (dh, _) = (_make(r, c, "bf16", 50 + i, s) for i, (r, c, s) in enumerate(
        ((T, D, 1.0), (F, D, D ** -0.5), (F, D, D ** -0.5), (T, F, 0.25))))
    h0, saved0 = hf.gated_forward(x, wg, wu, ckpt=(4, 3))
    d0 = hf.gated_backward(dh, saved0, wg, wu)
    nan, inf = float("nan"), float("inf")
    x1, w1 = x.clone(), wu.clone()
    x1[T - 1, 0], x1[255, D - 1], w1[F - 1, D - 1], w1[128, 0] = nan, nan, nan, nan
    h, saved = hf.gated_forward(x1, wg, w1, ckpt=(4, 3))
    _same(h0, h, [255, T - 1], [128, F - 1])
    for a, b, cols in ((saved0.gate, saved.gate, []), (saved0.up, saved.up, [128, F - 1])):
        a, b = (hf.block_unpack(*s, F, (4, 3)) for s in (a, b))
        for c in cols:   # (it may have been its group's largest: the group's other values may change)
            assert b[:, c].isnan().all()
            a[:, c // 32 * 32:c // 32 * 32 + 32] = b[:, c // 32 * 32:c // 32 * 32 + 32] = 0.0
        a[[255, T - 1]], b[[255, T - 1]] = 0.0, b[[255, T - 1]].nan_to_num(nan=0.0)
        assert torch.equal(a, b)
    # a token's NaN in dh: its row of dx, and of the weights' gradients the row of its place
    dh1 = dh.clone()
    dh1[T - 1, F - 1], dh1[256, 0] = nan, inf
    dx, dwg, dwu = hf.gated_backward(dh1, saved0, wg, wu)
    _same(d0[0], dx, [T - 1, 256])
    _same(d0[1], dwg, [F - 1, 0])
    _same(d0[2], dwu, [F - 1, 0])
    # one in x's blocks: a column of the weights' gradients
    x2 = x.clone()
    x2[T - 1, D - 1], x2[0, 0] = nan, nan
    dx, dwg, dwu = hf.gated_backward(dh, saved0._replace(x=hf.block_pack(x2, (4, 3))), wg, wu)
    assert torch.equal(dx, d0[0])
    _same(d0[1][:, 32:D // 32 * 32], dwg[:, 32:D // 32 * 32])
    assert dwg[:, [0, D - 1]].isnan().all() and dwu[:, [0, D - 1]].isnan().all()
    assert dwg[:, 1:D - 1].isfinite().all() and dwu[:, 1:D - 1].isfinite().all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,K,N,group,scale", [(20, 136, 8200, 32, "pow2"), (64, 264, 8193, 64, "bf16"),
                                               (33, 1040, 8200, 128, "f32"), (70, 72, 9001, 32, "f32")])
def test_w4_tiles(T, K, N, group, scale, dtype):
    hf = need_gpu()
    say("isolation, w4", T, K, N, group, scale, dtype)
    cg, sg, w = _weights(hf, N, K, group, scale, 51)
    cu, su, _ = _weights(hf, N, K, group, scale, 52)
    x = _x(T, K, dtype, 53).clone()
    y0, h0 = hf.w4_linear(x, cg, sg, group=group), hf.w4_gated(x, cg, sg, cu, su, group=group)
    x1, s1 = x.clone(), sg.clone()
    x1[T - 1, K - 1], x1[3, 0] = float("nan"), float("nan")
    _same(y0, hf.w4_linear(x1, cg, sg, group=group), [3, T - 1])
    _same(h0, hf.w4_gated(x1, cg, sg, cu, su, group=group), [3, T - 1])
    # a scale: its row alone; the sums of a wave's other rows may be formed in another order
    s1[N - 1, s1.shape[1] - 1] = s1[77, 0] = 255 if scale == "pow2" else float("nan")
    y = hf.w4_linear(x, cg, s1, group=group)
    assert y[:, [77, N - 1]].isnan().all()
    keep = torch.ones(N, dtype=torch.bool)
    keep[[77, N - 1]] = False
    a, b = y0.double().cpu()[:, keep], y.double().cpu()[:, keep]
    size = x.double().cpu().abs() @ torch.from_numpy(w).abs().T[:, keep]
    assert ((a - b).abs() <= UNIT[dtype] * a.abs() + 2 * (K + 4) * EPS * size + TINY[dtype]).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [136, 264])
def test_w4_tiles_every_power_of_two(K, group, dtype):
    """Scale bytes from 0 to 255, one a row, alone and among ordinary ones, with K that ends inside a
    step: weights picked one by one are the code's value times the scale, rounded once."""
    hf = need_gpu()
    T, N = 20, 8200
    say("w4 tiles, powers of two", K, group, dtype)
    rng = np.random.default_rng(54)
    packed = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    groups = -(-K // group)
    b = np.repeat((np.arange(N) % 256)[:, None], groups, 1)
    b[N // 2:, 1::2] = 127
    f = np.where(b == 255, np.nan, np.exp2(b - 127.0))
    with np.errstate(invalid="ignore", over="ignore"):
        w = ref.unpack(ref.nibbles(packed, K), f, (2, 1), group).astype(np.float32)
    packed, scales = torch.from_numpy(packed).cuda(), torch.from_numpy(b.astype(np.uint8)).cuda()
    nan = torch.from_numpy(np.isnan(f).any(1))
    for k0 in (0, 17, 31, 64, 120, K - T):
        k0 = min(k0, K - T)
        x = torch.zeros(T, K, dtype=TYPES[dtype])
        x[torch.arange(T), k0 + torch.arange(T)] = 1.0
        y = hf.w4_linear(x.cuda(), packed, scales, group=group).cpu()
        want = torch.from_numpy(w[:, k0:k0 + T].T.copy()).to(TYPES[dtype])
        assert y[:, nan].isnan().all()
        assert torch.equal(y[:, ~nan], want[:, ~nan])
