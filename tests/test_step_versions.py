"""What autograd is told of tensors that a call writes: those and no others (CPU: the library and the GPU are stand-ins)."""
import pytest
import torch

from paper_2007_06563_amd import hobflops as hf
from test_devices import Gpu, _gpu, calls  # noqa: F401

f32 = torch.float32


@pytest.fixture
def gpu(calls, monkeypatch):
    monkeypatch.setattr(hf, "_get_device", lambda t: t.device.index)
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **k: zeros(*a, **k).as_subclass(Gpu))
    return calls


def _versions(ts):
    return [None if t is None else t._version for t in ts]


@pytest.mark.parametrize("given", [(0, 2), (1,), (0, 1, 2), ()])
@pytest.mark.parametrize("copied", [(), (0, 1), (0, 1, 2)])
def test_a_step_changes_what_has_a_gradient(gpu, given, copied):
    params = [_gpu(40, dtype=f32) for _ in range(3)]
    copies = [_gpu(40) if i in copied else None for i in range(3)]
    grads = [_gpu(40) if i in given else None for i in range(3)]
    state = hf.adamw_state(params)
    before = _versions(params), _versions(copies), _versions([g for g in grads if g is not None])
    hf.adamw(params, grads, state, 1, copies=copies)
    for i in range(3):
        assert params[i]._version == before[0][i] + (i in given)
        if i in copied:
            assert copies[i]._version == before[1][i] + (i in given)
    assert _versions([g for g in grads if g is not None]) == before[2]


def test_a_frozen_weight_keeps_what_autograd_saved(gpu):
    """A weight without a gradient may be part of a graph that a step of the others stands in the middle of."""
    frozen, other = torch.ones(8).requires_grad_(), _gpu(8, dtype=f32)
    loss = (frozen * frozen).sum()
    view = frozen.detach().as_subclass(Gpu)      # the same memory and version
    hf.adamw([view, other], [None, _gpu(8, dtype=f32)], hf.adamw_state([view, other]), 1)
    loss.backward()
    assert torch.equal(frozen.grad, torch.full((8,), 2.0))


def _pair(rows, cols):
    return _gpu(rows, cols), _gpu(rows, cols)


OUT = {
    "layer_norm": lambda x, out: hf.layer_norm(x, out=out),
    "linear": lambda x, out: hf.linear(x, _gpu(64, 64), out=out),
    "gated_forward": lambda x, out: hf.gated_forward(x, _gpu(64, 64), _gpu(64, 64), out=out),
    "w4_linear": lambda x, out: hf.w4_linear(x, _gpu(64, 32, dtype=torch.uint8), _gpu(64, 2, dtype=torch.uint8), out=out),
    "w4_gated": lambda x, out: hf.w4_gated(x, *[_gpu(64, n, dtype=torch.uint8) for n in (32, 2, 32, 2)], out=out),
    "block_unpack": lambda x, out: hf.block_unpack(_gpu(4, 64, dtype=torch.uint8), _gpu(4, 2, dtype=torch.uint8), 64, (4, 3),
                                                   out=out),
}


@pytest.mark.parametrize("name", OUT)
def test_a_given_output_is_changed(gpu, name):
    """What autograd has saved of an output that the caller gives is not there any more."""
    x, out = _pair(4, 64)
    before = x._version, out._version
    assert OUT[name](x, out) is out
    assert (x._version, out._version) == (before[0], before[1] + 1)


@pytest.mark.parametrize("call", [lambda x: hf.layer_norm(x, out=x),
                                  lambda x: hf.linear(_gpu(4, 64), _gpu(64, 64), residual=x, out=x)])
def test_a_call_in_place_is_seen(gpu, call):
    x = torch.ones(4, 64, dtype=torch.bfloat16).requires_grad_()
    loss = (x * x).sum()
    call(x.detach().as_subclass(Gpu))             # the same memory and version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_columns_of_a_wider_output(gpu):
    """A view's version is its base's."""
    wide = _gpu(4, 128)
    before = wide._version
    hf.layer_norm(_gpu(4, 64), out=wide[:, 64:])
    assert wide._version == before + 1


@pytest.mark.parametrize("given", [(), ("codes",), ("scales",), ("codes", "scales")])
def test_given_blocks_are_changed(gpu, given):
    x, blocks = _gpu(4, 64), dict(codes=_gpu(4, 64, dtype=torch.uint8), scales=_gpu(4, 2, dtype=torch.uint8))
    before = {k: t._version for k, t in blocks.items()}
    hf.block_pack(x, (4, 3), **{k: blocks[k] for k in given})
    assert all(t._version == before[k] + (k in given) for k, t in blocks.items())


@pytest.mark.parametrize("fmt", [None, (4, 3)])
def test_a_steps_states_are_changed(gpu, fmt):
    p = [_gpu(40, dtype=f32)]
    state = hf.adamw_state(p, fmt)
    parts = [state.m, state.v] if fmt is None else [*state.m, *state.v]
    before = _versions(parts)
    hf.adamw(p, [_gpu(40)], state, 1)
    assert _versions(parts) == [v + 1 for v in before]
