"""The example's autograd function: gated_backward's gradients, and an error for a second derivative."""
import importlib.util
import os
import warnings

import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def _case():
    g = torch.Generator(device="cuda").manual_seed(61)
    x, wg, wu = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((5, 64), (96, 64), (96, 64)))
    return x, wg, wu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_function_has_first_derivatives_only():
    hf = need_gpu()
    m = _example()
    x, wg, wu = (t.requires_grad_() for t in _case())
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        h = m.Gated.apply(x, wg, wu)
    dh = torch.randn_like(h)
    got = torch.autograd.grad(h, (x, wg, wu), dh, retain_graph=True)
    with torch.no_grad():
        _, saved = hf.gated_forward(x, wg, wu, ckpt=(4, 3))
        want = hf.gated_backward(dh, saved, wg, wu)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dx, = torch.autograd.grad(h.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (h.float().sum() + dx.float().square().sum()).backward()
