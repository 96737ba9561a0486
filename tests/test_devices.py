"""Every call of the binding runs with its tensors' device as the current one, on that device's stream: the
default stream is whichever device is current (CPU: the library and the GPU's state are stand-ins)."""
import types

import pytest
import torch

from paper_2007_06563_amd import hobflops as hf


class Gpu(torch.Tensor):
    """A host tensor that says it is on cuda:1."""
    is_cuda = True
    device = torch.device("cuda:1")


def _gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(Gpu)


@pytest.fixture
def calls(monkeypatch):
    state = types.SimpleNamespace(device=0, seen=[])

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if name == "hobflops_plane_words":
                    args[3]._obj.value = args[0] * (-(-args[1] // 32)) * (3 + args[2].wE + args[2].wF)
                elif name == "hobflops_gated_workspace":
                    args[2]._obj.value = 64
                else:
                    stream = getattr(args[-1], "value", args[-1])
                    state.seen.append((name, state.device, stream))
                return 0
            return call

    class Current:
        def __init__(self, device):
            self.device = torch.device(device).index if not isinstance(device, int) else device

        def __enter__(self):
            self.before, state.device = state.device, self.device

        def __exit__(self, *a):
            state.device = self.before

    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).as_subclass(Gpu))
    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state.device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state.device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 1000 + i)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: types.SimpleNamespace(
        cuda_stream=1000 + (state.device if d is None else torch.device(d).index)))
    monkeypatch.setattr(hf, "lib", Lib)
    return state


def _saved(T, D, F):
    def blocks(c):
        return _gpu(T, c, dtype=torch.uint8), _gpu(T, -(-c // 32), dtype=torch.uint8)
    return hf.GatedSaved(blocks(D), blocks(F), blocks(F), hf.fmt((4, 3)))


def _planes(rows, cols, f):
    return _gpu(*hf.plane_shape(rows, cols, f), dtype=torch.int32)


F53, F54 = (5, 3), (5, 4)
DESC = (1, 8, 8, 4, 8, 3, 3, 1, 1, F53, F54, F54)
CALLS = {
    "pack": lambda: hf.pack(_gpu(4, 32, dtype=torch.float32), F53),
    "pack_batch": lambda: hf.pack_batch([_gpu(4, 32, dtype=torch.float32)], F53),
    "unpack": lambda: hf.unpack(_planes(4, 32, F53), 4, 32, F53),
    "conv2d": lambda: hf.conv2d(_planes(64, 4, F53), _planes(36, 8, F53), hf.conv_desc(*DESC)),
    "conv2d_on_values": lambda: hf.conv2d_on_values(_planes(64, 4, F53), _planes(36, 8, F53),
                                                    hf.conv_desc(*DESC), hf.TILE_32X32),
    "muladd": lambda: hf.muladd(*[_planes(1, 32, F53)] * 3, 32, F53, F54),
    "avgpool": lambda: hf.avgpool(_planes(4, 32, F53), 1, 2, 2, 32, F53, F54, F54),
    "block_pack": lambda: hf.block_pack(_gpu(4, 64), (4, 3)),
    "block_unpack": lambda: hf.block_unpack(_gpu(4, 64, dtype=torch.uint8), _gpu(4, 2, dtype=torch.uint8),
                                            64, (4, 3)),
    "gated_forward": lambda: hf.gated_forward(_gpu(4, 64), _gpu(96, 64), _gpu(96, 64)),
    "gated_forward_ckpt": lambda: hf.gated_forward(_gpu(4, 64), _gpu(96, 64), _gpu(96, 64), ckpt=(4, 3)),
    "gated_backward": lambda: hf.gated_backward(_gpu(4, 96), _saved(4, 64, 96), _gpu(96, 64), _gpu(96, 64)),
    "w4_linear": lambda: hf.w4_linear(_gpu(2, 64), _gpu(8, 32, dtype=torch.uint8), _gpu(8, 2)),
    "w4_gated": lambda: hf.w4_gated(_gpu(2, 64), *[_gpu(8, 32, dtype=torch.uint8), _gpu(8, 2)] * 2),
}


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("name", list(CALLS))
def test_runs_on_its_tensors_device(calls, name, current):
    calls.device = current
    CALLS[name]()
    assert calls.seen and all(d == 1 and s == 1001 for _, d, s in calls.seen), calls.seen
    assert calls.device == current
