"""What the search's recovery judges by: the first model's own answers, features that the classifier makes them of, and the share that the tuning leaves, computed apart
from it in 64 bits."""
import pytest
import torch

from paper_2207_01260_amd import binding as B
from paper_2207_01260_amd import search as psearch
from paper_2207_01260_amd.recover import AdaptedLinear

pytestmark = pytest.mark.gpu

STEPS = 3


def tuned64(layer, x, ids, teacher, steps, rate, temperature=2.0):
    """Logits of a layer after `steps` of gradient descent on the mean of T^2 KL(teacher's list, softmax of the row), in 64 bits on the codes' own product."""
    base = B.cprune_mx4_linear(x, layer.codes, layer.scales, layer.bias).double()
    a, b, x, s = layer.a[0].double(), layer.b[0].double(), x.double(), float(layer.scale[0])
    p = torch.softmax(teacher.double() / temperature, dim=1)
    for _ in range(steps):
        hidden = s * x @ a.t()
        slope = torch.softmax((base + hidden @ b.t()) / temperature, dim=1)
        slope = temperature * slope.scatter_add(1, ids.long(), -p) / len(x)
        a, b = a - rate * (s * slope @ b).t() @ x, b - rate * slope.t() @ hidden
    return base + s * x @ a.t() @ b.t()


@pytest.mark.parametrize("net,dtype", [("vgg16", B.F32), ("resnet18", B.F32), ("mobilenetv2", B.F32), ("mnasnet", B.F32), ("vgg16", B.BF16), ("mobilenetv2", B.F16)])
def test_search_with_recovery(net, dtype):
    ds, start, _, log = psearch.run(net, batch=16, dtype=dtype, iterations=2, beta=10.0, recover=STEPS)
    first = ds._state(start)
    # the teacher is the model that the search began with
    values, ids = B.cprune_top_logits(first["logits"], min(8, first["logits"].shape[1]))
    assert torch.equal(ds.teacher[0], values) and torch.equal(ds.teacher[1], ids)
    judged = [a for _, _, _, a, verdict in log if verdict in ("accepted", "inaccurate")]
    models = [m for m, _, _, _ in ds.trace]
    assert models[0] == start and set(judged) <= {ds.accuracy(m) for m in models[1:]}
    # (the tasks that a network's search begins with may have nothing to prune: a candidate for certain)
    some = ds.prunable[len(ds.prunable) // 2]
    models.append({**start, some: max(1, start[some] - 16)})
    u = {B.F32: 2.0 ** -24, B.F16: 2.0 ** -11, B.BF16: 2.0 ** -8}[dtype]
    for model in models:
        st = ds._state(model)
        w, bias = st["classifier"]
        x = st["features"]
        assert x.shape == (16, w.shape[1])
        # logits are the classifier's answer to the features: sums of c products in 32 bits, weights and features rounded to the type once
        product, size = x.double() @ w.double().t() + bias.double(), x.double().abs() @ w.double().abs().t() + bias.double().abs()
        off = (size * (4 * u + (32 + 2 * w.shape[1] ** 0.5) * 2.0 ** -24)) + u * product.abs()
        assert ((st["logits"].double() - product).abs() <= off).all()
        layer = AdaptedLinear(w, bias)
        z = tuned64(layer, x, ids, values, STEPS, 0.5 / max(1.0, float(x.float().square().mean())))
        top = z.topk(2, dim=1).values
        near = (top[:, 0] - top[:, 1]) <= 16 * u * z.abs().amax(dim=1)      # (rows whose answer a rounding may change)
        share = (z.argmax(dim=1) == ids[:, 0]).double().mean()
        assert abs(float(share) - ds.accuracy(model)) <= float(near.double().mean()), model
