"""Adapters beside which one side of the projection has fewer numbers than a vector (8 of 16 bits, 4 of 32): a pruned classifier of two classes, a layer behind a handful
of channels.  Bounds as in the tests of the adapters."""
import pytest
import torch

import test_gpu_adapter as adapter
from test_gpu_many_rows import poison
from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu

# (rows, k, c_out, rank, adapters): the wide side a vector and one more, odd past one and past several work-groups of columns, whole; each rank's form
SHAPES = [(70, 83, 5, 6, 2), (70, 20, 3, 3, 4), (70, 342, 2, 8, 1), (70, 5, 45, 5, 2), (70, 130, 3, 33, 3), (200, 3, 257, 20, 3), (130, 5, 203, 9, 3), (90, 7, 9, 2, 2),
          (90, 5, 3, 1, 1), (300, 1, 1030, 100, 2), (1000, 515, 1, 16, 5), (70, 128, 4, 8, 2), (33, 4, 136, 12, 2), (5, 3, 45, 5, 2), (2000, 2, 77, 70, 4)]


@pytest.mark.parametrize("order", ["one", "runs", "mixed"])
@pytest.mark.parametrize("dtype", adapter.TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_one_side_thin(shape, dtype, order):
    m = adapter.make(shape, dtype, order, seed=20)
    poison()
    got, grads = adapter.check(m)
    full = grads[1:]
    alone = B.cprune_adapter_linear_backward(m["dy"], m["x"], got[1], m["a"], m["b"], m["which"], m["scale"], want_dx=False)
    assert alone[0] is None and all(torch.equal(p, q) for p, q in zip(full, alone[1:]))


@pytest.mark.parametrize("dtype", adapter.TYPES)
@pytest.mark.parametrize("shape", [(70, 83, 5, 6, 2), (70, 5, 133, 5, 2)])
def test_one_side_thin_of_wider_rows(shape, dtype):
    """What lies behind a row, NaN here, is not the row's."""
    m = adapter.make(shape, dtype, "mixed", seed=21, wide=9)
    rows, k, c_out = shape[:3]
    for name, c in (("x", k), ("dy", c_out), ("base", c_out), ("dx_base", k)):
        wide = m[name].new_full((rows, c + 9), float("nan"))
        wide[:, :c] = m[name]
        m[name] = wide[:, :c]
    adapter.check(m)
