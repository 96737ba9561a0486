"""The gated block's operators beside torch's autograd: they record nothing and say so."""
import warnings

import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def _case():
    g = torch.Generator(device="cuda").manual_seed(61)
    x, wg, wu = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((5, 64), (96, 64), (96, 64)))
    return x, wg, wu


@pytest.mark.parametrize("which", [0, 1, 2])
def test_a_lost_gradient_is_told(which):
    hf = need_gpu()
    t = list(_case())
    t[which].requires_grad_()
    want = hf.gated_forward(*(v.detach() for v in t))
    with pytest.warns(UserWarning, match="no gradient"):
        h = hf.gated_forward(*t)
    assert not h.requires_grad and torch.equal(h, want)
    with pytest.warns(UserWarning, match="no gradient"):
        hf.gated_forward(*t, ckpt=(4, 3))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            hf.gated_forward(*t)
        hf.gated_forward(*(v.detach() for v in t))


def test_a_lost_gradient_is_told_by_4_bit_products():
    hf = need_gpu()
    x, wg, wu = _case()
    g, u = (hf.block_pack(w, (2, 1)) for w in (wg, wu))
    x.requires_grad_()
    with pytest.warns(UserWarning, match="no gradient"):
        hf.w4_linear(x, *g)
    with pytest.warns(UserWarning, match="no gradient"):
        hf.w4_gated(x, *g, *u)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            hf.w4_gated(x, *g, *u)
