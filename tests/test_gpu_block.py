"""Blocks of narrow floats on the GPU against a plain 64-bit reference: codes, scales and values are
compared bit for bit (the format defines them)."""
import numpy as np
import pytest
import torch

import narrow_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F8 = [(4, 3), (5, 2)]


def _matrix(rows, cols, dtype, seed, gap=0, offset=0):
    """Values of widely spread groups, as a part of a wider tensor at an offset."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols + gap), generator=g)
    spread = 6 if dtype == "f16" else 30
    x = x * torch.exp2(torch.randint(-spread, spread, (rows, 1 + (cols + gap) // 32), generator=g)
                       .float()).repeat_interleave(32, 1)[:, :cols + gap]
    flat = torch.zeros(rows * (cols + gap) + offset, dtype=TYPES[dtype])
    flat[offset:] = x.to(TYPES[dtype]).reshape(-1)
    return flat.cuda()[offset:].view(rows, cols + gap)[:, :cols]


def _check8(hf, x, f):
    codes, scales = hf.block_pack(x, f)
    want, factors = ref.pack(x.double().cpu().numpy(), f)
    assert np.array_equal(scales.cpu().numpy(), np.log2(factors).astype(int) + 127)
    got = codes.cpu().numpy().astype(np.int64)
    nan = np.isnan(ref.decode(want, f))
    assert np.array_equal(np.isnan(ref.decode(got, f)), nan)
    assert np.array_equal(got[~nan], want[~nan])
    values = ref.unpack(want, factors, f)
    for t in (torch.float32, torch.bfloat16, torch.float16):
        back = hf.block_unpack(codes, scales, x.shape[1], f, dtype=t)
        exp = torch.from_numpy(values).to(torch.float32).to(t)
        assert torch.equal(torch.nan_to_num(back.cpu().float(), nan=0.5, posinf=1e39, neginf=-1e39),
                           torch.nan_to_num(exp.float(), nan=0.5, posinf=1e39, neginf=-1e39))
        assert torch.equal(torch.signbit(back.cpu()) | back.cpu().isnan(),
                           torch.signbit(exp) | exp.isnan())


@pytest.mark.parametrize("f", F8)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,gap,offset", [(1, 1, 0, 0), (1, 32, 0, 0), (3, 33, 0, 0),
                                                  (5, 64, 8, 0), (7, 100, 3, 1), (2, 8, 0, 1),
                                                  (65, 520, 0, 0), (33, 257, 7, 3)])
def test_pack8(f, dtype, rows, cols, gap, offset):
    hf = need_gpu()
    say("pack8", f, dtype, rows, cols, gap, offset)
    _check8(hf, _matrix(rows, cols, dtype, 7 * rows + cols, gap, offset), f)


@pytest.mark.parametrize("f", F8)
def test_pack8_every_step(f):
    """Groups whose values are the format's midpoints and steps, from below its smallest to its
    largest, and groups whose largest value stands at the limit where the scale changes."""
    hf = need_gpu()
    v = ref.code_values(f)
    mid = (v[1:] + v[:-1]) / 2
    near = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(np.inf)),
                           np.nextafter(mid.astype(np.float32), np.float32(0))]).astype(np.float32)
    near = np.concatenate([near, -near])
    near = np.concatenate([near, np.zeros(-len(near) % 31, np.float32)]).reshape(-1, 31)
    # a value of the largest code in every group pins the scale
    x = np.concatenate([near, np.full((len(near), 1), v[-1], np.float32)], 1)
    lim = np.float32(ref.limit(f)[0])
    edge = np.array([lim, np.nextafter(lim, np.float32(0)), np.nextafter(lim, np.float32(np.inf)),
                     v[-1], 2 * v[-1], 1.0], np.float32)
    top = np.zeros((len(edge), 32), np.float32)
    top[:, 5], top[:, 6] = edge, edge / 3
    for scale in (1.0, 2.0 ** -100, 2.0 ** 90):
        _check8(hf, torch.from_numpy(np.concatenate([x, top]) * np.float32(scale)).cuda(), f)


@pytest.mark.parametrize("f", F8)
def test_pack8_special(f):
    """Zeros of both signs, subnormals, the largest values, infinities and NaN, alone and among
    others: what is not finite does not change the group's scale."""
    hf = need_gpu()
    inf, nan = np.inf, np.nan
    rows = [[0.0, -0.0], [1e-45, -1e-45], [1e-38, 3e-39], [3.4e38, -3.3e38, 1.0], [inf, 1.0, -2.0],
            [-inf, inf], [nan, 3.0], [nan], [nan, inf, -0.0, 5e-324 * 0], [2.0 ** -100, 1.0],
            [2.0 ** -120, -2.0 ** -126]]
    x = np.zeros((len(rows), 40), np.float32)
    for i, r in enumerate(rows):
        x[i, 3:3 + len(r)] = r
        x[i, 39] = r[0]
    _check8(hf, torch.from_numpy(x).cuda(), f)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scale", ["pow2", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,gap,offset", [(1, 1, 0, 0), (3, 33, 0, 0), (5, 256, 0, 0),
                                                  (4, 131, 5, 1), (6, 130, 6, 0)])
def test_pack4(group, scale, rows, cols, gap, offset):
    hf = need_gpu()
    say("pack4", group, scale, rows, cols, gap, offset)
    x = _matrix(rows, cols, "f32", rows + cols, gap, offset)
    if cols > 100:
        x[1, 3], x[2, cols - 1] = float("nan"), float("inf")
    x[0] = 0.0
    kind = {"pow2": hf.SCALE_POW2, "bf16": hf.SCALE_BF16, "f32": hf.SCALE_F32}[scale]
    codes, scales = hf.block_pack(x, (2, 1), group=group, scale=kind)
    rnd = {"pow2": "pow2", "f32": lambda s: s,
           "bf16": lambda s: torch.tensor(s).bfloat16().float().item()}[scale]
    want, factors = ref.pack(x.double().cpu().numpy(), (2, 1), group, rnd)
    got = ref.nibbles(codes.cpu().numpy(), cols)
    fin = ~np.isnan(np.repeat(factors, group, 1)[:, :cols])
    assert np.array_equal(got[fin], want[fin])
    sc = scales.cpu()
    have = (np.where(sc.numpy() == 255, np.nan, np.exp2(sc.double().numpy() - 127))
            if scale == "pow2" else sc.double().numpy())
    assert np.array_equal(have, factors, equal_nan=True)
    back = hf.block_unpack(codes, scales, cols, (2, 1), group=group)
    exp = torch.from_numpy(ref.unpack(want, factors, (2, 1), group)).float()
    assert np.array_equal(back.cpu().numpy()[fin], exp.numpy()[fin])
    assert np.isnan(back.cpu().numpy()[~fin]).all()
    if cols % 2:
        assert not (codes[:, -1] >> 4).any()


def test_unpack_every_code():
    """All codes of every format under scales from the smallest to NaN."""
    hf = need_gpu()
    for f in ((4, 3), (5, 2)):
        codes = torch.arange(256, dtype=torch.uint8).repeat(5, 1).cuda()
        sc = torch.tensor([0, 17, 127, 200, 255], dtype=torch.uint8).repeat(8, 1).t().contiguous()
        got = hf.block_unpack(codes, sc.cuda(), 256, f).cpu().numpy()
        s = np.array([2.0 ** -127, 2.0 ** -110, 1.0, 2.0 ** 73, np.nan])
        with np.errstate(invalid="ignore"):
            want = (ref.decode(np.arange(256), f)[None] * s[:, None]).astype(np.float32)
        assert np.array_equal(got, want, equal_nan=True)
    codes = torch.arange(256, dtype=torch.uint8).reshape(1, 256).cuda()
    sc = torch.full((1, 16), 127, dtype=torch.uint8).cuda()
    got = hf.block_unpack(codes, sc, 512, (2, 1)).cpu().numpy()
    assert np.array_equal(got, ref.decode(ref.nibbles(np.arange(256)[None], 512), (2, 1)))


def test_empty_and_output_parts():
    """No rows or no columns; outputs that are parts of wider tensors leave the rest as it is; a
    stream other than the default one."""
    hf = need_gpu()
    for shape in ((0, 32), (3, 0)):
        codes, scales = hf.block_pack(torch.zeros(shape, device="cuda"), (4, 3))
        assert hf.block_unpack(codes, scales, shape[1], (4, 3)).shape == shape
    x = _matrix(9, 70, "bf16", 3)
    wide = torch.full((9, 90), 7.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        codes, scales = hf.block_pack(x, (4, 3))
        hf.block_unpack(codes, scales, 70, (4, 3), out=wide[:, 3:73])
    s.synchronize()
    want, factors = ref.pack(x.double().cpu().numpy(), (4, 3))
    exp = torch.from_numpy(ref.unpack(want, factors, (4, 3))).bfloat16()
    assert torch.equal(wide[:, 3:73].cpu(), exp)
    assert (wide[:, :3] == 7).all() and (wide[:, 73:] == 7).all()
