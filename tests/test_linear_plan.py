"""The shapes at which the linear layer's kernels are tested reach all of them (CPU: the plan alone)."""
import os
import tempfile

import pytest

import linear_shapes


@pytest.fixture(scope="module")
def plans():
    with tempfile.TemporaryDirectory() as folder:
        return linear_shapes.plans(linear_shapes.SHAPES, folder)


def test_every_forward_kernel_is_reached(plans):
    seen = {f for f, _ in plans}
    assert {f"direct{i}" for i in range(6)} <= seen
    tiles = {(f.split()[0], frozenset(f.split()[1:])) for f in seen if f.startswith("forward")}
    for kind in (f"forward{i}" for i in range(5)):
        have = [marks for name, marks in tiles if name == kind]
        for marks in (set(), {"parts"}, {"tail"}, {"parts", "tail"}, {"x", "w"}):
            # (one operand copied or none for the first four)
            assert any(m - {"x", "w"} == marks - {"x", "w"} and marks <= m for m in have), (kind, marks)
        for copied in ("x", "w"):
            assert any(copied in m and "tail" in m for m in have), (kind, copied)


def test_every_product_of_the_gradients_is_reached(plans):
    seen = [b for _, b in plans]
    for product in ("dx", "dw"):
        for kind in range(3):
            for parts in (True, False):
                assert any(f"{product}{kind}" in b and (f"{product}{kind} parts" in b) == parts for b in seen), (product, kind, parts)
    for kind in range(3):
        assert any("joint" in b and f"dx{kind}" in b for b in seen), kind
    for first, second in ((0, 1), (1, 0), (0, 2), (2, 0), (2, 1)):
        assert any("apart" in b and f"dx{first}" in b and f"dw{second}" in b for b in seen), (first, second)
    for copied in ("dz", "x", "w"):
        assert any(copied in b.split() for b in seen) and any(copied not in b.split() for b in seen)
