"""hidden and g reach y and dx with all of their 24 bits, also beside 16-bit operands: seen where what they make cancels.

Bounds as in the tests of the adapters, without what two parts of 8 bits would be short: every product is exact, and three parts, six products beside fp16, make sums of up to
six times as many terms."""
import pytest
import torch

import test_gpu_adapter as adapter
from test_gpu_adapter import B, E, near, wide64

pytestmark = pytest.mark.gpu


def whole(monkeypatch, rank):
    more = 2 * ((6 * rank) ** 0.5 - rank ** 0.5) * E
    monkeypatch.setattr(adapter, "SHORT", {t: more for t in adapter.TYPES})


@pytest.mark.parametrize("order", ["one", "mixed"])
@pytest.mark.parametrize("dtype", adapter.TYPES)
@pytest.mark.parametrize("rows,k,c_out,rank", [(1500, 4, 40, 2, ), (40, 6, 300, 4), (700, 5, 33, 8), (300, 8, 100, 40), (300, 8, 72, 72)])
def test_answers_that_cancel(rows, k, c_out, rank, dtype, order, monkeypatch):
    """Ranks in pairs that differ by a small input's part alone, with opposite signs in B."""
    m = adapter.make((rows, k, c_out, rank, 3 if order == "mixed" else 1), dtype, order, seed=30)
    m["a"][:, 1::2] = m["a"][:, 0::2]
    m["a"][:, 1::2, 0] = 0
    m["b"][:, :, 1::2] = -m["b"][:, :, 0::2]
    m["x"][:, 0] *= 2.0 ** -12
    whole(monkeypatch, rank)
    y, bound, _, _ = adapter.forward64(m, B.ACT_NONE, base=False)
    near(B.cprune_adapter_linear(m["x"], m["a"], m["b"], m["which"], m["scale"]), y, bound, "y")


@pytest.mark.parametrize("order", ["one", "mixed"])
@pytest.mark.parametrize("dtype", adapter.TYPES)
@pytest.mark.parametrize("rows,k,c_out,rank", [(1500, 40, 4, 2), (40, 300, 6, 4), (700, 33, 5, 8), (300, 100, 8, 40), (300, 72, 8, 72)])
def test_gradients_that_cancel(rows, k, c_out, rank, dtype, order, monkeypatch):
    """The same of the input's gradient: pairs that differ by a small gradient's part, with opposite signs in A."""
    m = adapter.make((rows, k, c_out, rank, 3 if order == "mixed" else 1), dtype, order, seed=31)
    m["b"][:, :, 1::2] = m["b"][:, :, 0::2]
    m["b"][:, 0, 1::2] = 0
    m["a"][:, 1::2] = -m["a"][:, 0::2]
    m["dy"][:, 0] *= 2.0 ** -12
    whole(monkeypatch, rank)
    hidden = torch.zeros(rows, rank, device="cuda")
    (dx, bound), _, _ = adapter.backward64(m, hidden, base=False)
    got = B.cprune_adapter_linear_backward(m["dy"], m["x"], hidden, m["a"], m["b"], m["which"], m["scale"])
    near(got[0], dx, bound, "dx")


@pytest.mark.parametrize("dtype", adapter.TYPES)
@pytest.mark.parametrize("rows", [1, 20, 100])
def test_one_bit_that_is_left(rows, dtype):
    """1 + 2^-10 + 2^-20 less 1 + 2^-10, exactly, forwards and backwards."""
    x = torch.tensor([1, 2.0 ** -10, 2.0 ** -20], device="cuda").expand(rows, 3).contiguous().to(dtype)
    a = torch.tensor([[[1, 1, 1], [1, 1, 0]]], device="cuda").to(dtype)
    b = torch.tensor([[[1, -1], [-2, 2]]], device="cuda").to(dtype)
    y, hidden = B.cprune_adapter_linear(x, a, b, want_hidden=True)
    assert (wide64(y) == [2.0 ** -20, -2.0 ** -19]).all()
    # the same factors the other way round: dy against A's transpose, then B's
    dx, _, _ = B.cprune_adapter_linear_backward(x, y, hidden, b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous())
    assert torch.equal(dx, y)
