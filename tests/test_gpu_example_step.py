"""The example's block: its gradients are the operators', and a step changes what the next pass reads."""
import importlib.util
import os

import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_are_the_operators():
    hf = need_gpu()
    m = _example()
    g = torch.Generator(device="cuda").manual_seed(3)
    block = m.Block(72, 136, g)
    x = torch.randn(9, 72, generator=g, device="cuda").bfloat16().requires_grad_()
    dy = torch.randn(9, 72, generator=g, device="cuda").bfloat16()
    y = block(x)
    y.backward(dy)
    with torch.no_grad():
        scale, shift, gate, up, down, bias = block.copies
        n, kept = hf.layer_norm(x, scale, shift, save=True)
        h, saved = hf.gated_forward(n, gate, up, ckpt=m.E4M3)
        assert torch.equal(y, hf.linear(h, down, bias, residual=x))
        dh, ddown, dbias = hf.linear_backward(dy, h, down)
        dn, dgate, dup = hf.gated_backward(dh, saved, gate, up)
        dx, dscale, dshift = hf.layer_norm_backward(dn, x, kept, scale)
    for c, want in zip(block.copies, (dscale, dshift, dgate, dup, ddown, dbias)):
        assert torch.equal(c.grad, want)
    assert torch.equal(x.grad, dx + dy)   # autograd's own sum of the two paths
    block.step(1e-2)
    assert all(c.grad is None and torch.equal(c, w.bfloat16()) for c, w in zip(block.copies, block.weights))
    assert not torch.equal(block(x), y)


def test_no_second_derivatives():
    need_gpu()
    m = _example()
    block = m.Block(64, 96, torch.Generator(device="cuda").manual_seed(4))
    x = torch.randn(3, 64, device="cuda").bfloat16().requires_grad_()
    dx, = torch.autograd.grad(block(x).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.float().square().sum().backward()
