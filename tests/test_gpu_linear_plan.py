"""The linear layer at sizes that reach each of its kernels (which those are: test_linear_plan), against a plain 64-bit
reference, with the tolerances of the linear layer's own tests."""
import pytest

from gpu_util import need_gpu, say
from linear_shapes import SHAPES
from test_gpu_linear import _backward, _forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:3])))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_each_kernel(shape, dtype):
    hf = need_gpu()
    T, K, N, lds, off, act = shape
    lds = lds or (K, K, N, N)
    say("linear plan", shape, dtype)
    xs, ws, z = _forward(hf, T, K, N, dtype, act, True, dtype == "bf16", lds, off)
    _backward(hf, xs, ws, z, T, K, N, dtype, act, lds, off)
