"""What a forward norm writes beside y, mean and rstd, overlaps nothing else (CPU: no call reaches the GPU)."""
import ctypes

import pytest

from test_abi import hf  # noqa: F401  (the library, as a fixture)
from test_step_abi import _norm_desc


def _norm(hf, rows=4, **kw):
    """x, y (bfloat16 [rows][64]), weight, bias (float32 [64]), mean, rstd (float32 [rows])."""
    a = dict(x=0x100000, weight=0x200000, bias=0x300000, y=0x400000, mean=0x500000, rstd=0x600000)
    a.update(kw)
    return hf.lib().hobflops_layer_norm(_norm_desc(hf, rows=rows), *[ctypes.c_void_p(p) for p in a.values()], None)


@pytest.mark.parametrize("name", ["mean", "rstd"])
@pytest.mark.parametrize("of,last", [("x", 4 * 128 - 4), ("y", 4 * 128 - 4), ("weight", 252), ("bias", 252)])
def test_statistics_over_an_operand(hf, name, of, last):
    base = dict(x=0x100000, weight=0x200000, bias=0x300000, y=0x400000)[of]
    for at in (base, base + last, base - 12):   # the first value, the last one, the last statistic on the first value
        assert _norm(hf, **{name: at}) == -1, (name, of, hex(at))


def test_statistics_over_each_other(hf):
    for at in (0x500000, 0x50000c, 0x500000 - 12):
        assert _norm(hf, rstd=at) == -1
    assert _norm(hf, rows=1, rstd=0x500000) == -1
    assert _norm(hf, rows=1, mean=0x100000) == -1


def test_statistics_in_place(hf):
    """y over x is allowed, the statistics over both are not."""
    assert _norm(hf, y=0x100000, mean=0x100000) == -1
    assert _norm(hf, y=0x100000, rstd=0x1001fc) == -1
