"""Top logits, 4-bit products, adapters and the loss run together as a network's classifier is brought back.  Gradients against the formulas in 64 bits on the
forward pass's own numbers; whether a loss falls is no one's claim here.

Bounds: those of the single calls, u the type's half unit in the last place and e = 2^-24: dz is off by (3 d + 120) e of its probabilities and u of itself, da and db by
that of what they add up and by (36 + 2 sqrt(rows)) e of the magnitudes; g, within da, by (32 + 2 sqrt(c_out)) e more."""
import numpy as np
import pytest
import torch

from paper_2207_01260_amd import binding as B
from paper_2207_01260_amd import search as psearch
from paper_2207_01260_amd.recover import AdaptedLinear

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: E, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def wide64(t):
    return t.detach().cpu().double().numpy()


def softmax64(z):
    p = np.exp(z - z.max(axis=1, keepdims=True))
    return p / p.sum(axis=1, keepdims=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,c,classes,variants", [(64, 342, 10, 1), (37, 100, 1000, 3), (200, 83, 45, 4)])
def test_a_step(rows, c, classes, variants, dtype):
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, c, generator=g).to(dtype).cuda()
    w = (torch.randn(classes, c, generator=g) * c ** -0.5).cuda()
    bias = (0.1 * torch.randn(classes, generator=g)).cuda()
    which = None if variants == 1 else torch.randint(-1, variants, (rows,), generator=g).int().cuda()
    labels = torch.randint(classes, (rows,), generator=g).int().cuda()
    layer = AdaptedLinear(w, bias, rank=6, variants=variants, scale=1.5)
    layer.b += 0.05 * torch.randn(layer.b.shape, generator=g).cuda()
    values, ids = B.cprune_top_logits(B.cprune_fc(x, w.to(dtype), bias), min(8, classes))
    T, hard = 2.0, 0.25
    z, hidden = layer.forward(x, which, want_hidden=True)
    loss, da, db = layer.gradients(x, ids, values, labels, which, T, hard)
    z64, t64, i64 = wide64(z), wide64(values), ids.cpu().numpy()
    p = softmax64(t64 / T)
    q, one = softmax64(z64 / T), softmax64(z64)
    dz = (1 - hard) * T * q + hard * one
    far = z64.max(axis=1, keepdims=True) - z64
    err = ((1 - hard) * T * q * (3 * far / T + 120) + hard * one * (3 * far + 120)) * E
    for r in range(rows):
        np.add.at(dz[r], i64[r], -(1 - hard) * T * p[r])
        np.add.at(err[r], i64[r], (1 - hard) * T * p[r] * (3 * (t64[r].max() - t64[r]) / T + 120) * E)
        dz[r, int(labels[r])] -= hard
    # (each row's share, a rounded number, is between a half and one before the power of two is taken out)
    dz, err = dz / rows, (err + 2 * E * np.abs(dz)) / rows
    err += U[dtype] * (np.abs(dz) + err) + 2.0 ** -24 / 2 ** (rows.bit_length() - 1)
    log_q = z64 / T - z64.max(axis=1, keepdims=True) / T - np.log(np.exp((z64 - z64.max(axis=1, keepdims=True)) / T).sum(axis=1, keepdims=True))
    want = (1 - hard) * T * T * (p * (np.log(p) - np.take_along_axis(log_q, i64, 1))).sum(axis=1) - hard * np.log(one[np.arange(rows), labels.cpu().numpy()])
    size = T * T * (p * (200 + 4 * (t64.max(axis=1, keepdims=True) - t64)) * (np.abs(np.log(p)) + np.abs(np.take_along_axis(log_q, i64, 1)) + 1)).sum(axis=1) + 200 + 8 * far.max(axis=1)
    assert (np.abs(wide64(loss) - want) <= E * size).all()
    x64, h64, a64, b64 = wide64(x), wide64(hidden), wide64(layer.a.to(dtype)), wide64(layer.b.to(dtype))
    of = np.zeros(rows, int) if which is None else which.cpu().numpy()
    for v in range(variants):
        at = np.nonzero(of == v)[0]
        f = (36 + 2 * len(at) ** 0.5) * E
        want = dz[at].T @ h64[at]
        bound = err[at].T @ np.abs(h64[at]) + f * (np.abs(dz[at]).T @ np.abs(h64[at])) + 1e-30
        assert (np.abs(wide64(db[v]) - want) <= bound).all()
        gr = 1.5 * dz[at] @ b64[v]
        dg = 1.5 * (err[at] @ np.abs(b64[v]) + (32 + 2 * classes ** 0.5) * E * (np.abs(dz[at]) @ np.abs(b64[v])))
        want = gr.T @ x64[at]
        bound = dg.T @ np.abs(x64[at]) + f * (np.abs(gr).T @ np.abs(x64[at])) + 1e-30
        assert (np.abs(wide64(da[v]) - want) <= bound).all()
    before = layer.a.clone(), layer.b.clone()
    losses = layer.tune(x, ids, values, 2, 0.1, labels=labels, which=which, temperature=T, hard=hard)
    assert len(losses) == 2 and all(torch.isfinite(v) for v in losses)
    assert all((m != n).any() for m, n in zip(before, (layer.a, layer.b)))


def test_rows_without_a_variant_and_the_first_answer():
    """An adapter's second factor begins as 0: the layer answers as its codes do, and so do rows of no variant later on."""
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(20, 64, generator=g).cuda(), torch.randn(30, 64, generator=g).cuda()
    layer = AdaptedLinear(w, variants=2)
    plain = B.cprune_mx4_linear(x, layer.codes, layer.scales)
    which = torch.tensor([0, 1, -1, 5] * 5, dtype=torch.int32, device="cuda")
    assert torch.equal(layer.forward(x), plain) and torch.equal(layer.forward(x, which), plain)
    layer.b += 1
    z = layer.forward(x, which)
    alone = (which < 0) | (which > 1)
    assert torch.equal(z[alone], plain[alone]) and (z[~alone] != plain[~alone]).any(dim=1).all()


@pytest.mark.parametrize("net", ["vgg16", "resnet18"])
def test_search_with_recovery(net):
    """The search asks for the accuracy of its first model and of every candidate that is quick enough."""
    ds, start, final, log = psearch.run(net, batch=8, iterations=1, beta=10.0, recover=2)
    assert log and ds.teacher is not None
    assert 0.0 <= ds.accuracy(start) <= 1.0
    for _, l_m, l_t, a_s, verdict in log:
        assert verdict in ("accepted", "inaccurate", "slow", "exhausted")
        if verdict in ("accepted", "inaccurate"):
            assert l_m < l_t and 0.0 <= a_s <= 1.0
