"""The pointwise block in 4 bits: its answer, its gradients and its tuning, through the calls that make it up."""
import numpy as np
import pytest
import torch

from paper_2207_01260_amd import binding as B
from paper_2207_01260_amd import pointwise, synth

pytestmark = pytest.mark.gpu


def block_of(c_in, c_out, keep, groups, dtype, shape):
    w = torch.from_numpy(synth.tensor_normal((c_out, c_in, 1, 1), 311, c_out, std=(2.0 / c_in) ** 0.5)).cuda()
    block = pointwise.PointwiseBlock(w, keep, groups)
    block.weight = torch.from_numpy(synth.tensor_uniform((c_in,), 0.5, 1.5, 312)).cuda()
    block.bias = torch.from_numpy(synth.tensor_normal((c_in,), 313, std=0.2)).cuda()
    x = torch.from_numpy(synth.tensor_normal(shape + (c_in,), 314)).cuda().to(dtype)
    return w, block, x


def test_kept_filters_and_answer(orc):
    w, block, x = block_of(40, 64, 45, 5, torch.float32, (2, 6, 5))
    _, _, kept = orc.rank_filters(w.cpu().numpy(), 45)
    assert np.array_equal(block.kept.cpu().numpy(), kept)
    assert torch.equal(block.w, w[block.kept.long(), :, 0, 0])
    z = B.cprune_group_norm_act(x, 5, block.weight, block.bias, act=B.ACT_SILU)
    zc, zs = B.cprune_mx4_quantize(z)
    values = B.cprune_mx4_dequantize(zc, zs, 40).double() @ B.cprune_mx4_dequantize(block.codes, block.scales, 40).double().t()
    y = block.forward(x)
    assert y.shape == (2, 6, 5, 45)
    # (sums of 40 exact terms in fp32)
    assert torch.allclose(y.reshape(-1, 45).double(), values, rtol=2.0 ** -20, atol=2.0 ** -20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_against_the_formula(dtype):
    """In 64 bits through automatic differentiation, the codes' rounding of the activations passed through.  fp32: the chain's few hundred roundings of 2^-24;
    bf16: dy and dz are rounded to 2^-9 each, at random; either way an error of the gradients' lengths."""
    w, block, x = block_of(40, 64, 45, 5, dtype, (3, 7, 6))
    target = block.full(x) + 0.1
    error, dweight, dbias, dx = block.gradients(x, target)
    x64, w64, b64 = x.double().requires_grad_(), block.weight.double().requires_grad_(), block.bias.double().requires_grad_()
    v = x64.reshape(3, 42, 5, 8)
    mean, var = v.mean(dim=(1, 3), keepdim=True), v.var(dim=(1, 3), keepdim=True, correction=0)
    n = ((v - mean) / torch.sqrt(var + np.float64(np.float32(1e-5)))).reshape(3, 7, 6, 40) * w64 + b64
    z = n * torch.sigmoid(n)
    rounded = B.cprune_group_norm_act(x, 5, block.weight, block.bias, act=B.ACT_SILU)
    codes = B.cprune_mx4_dequantize(*B.cprune_mx4_quantize(rounded), 40).double().reshape(z.shape)
    z = z + (codes - z).detach()
    y = z @ B.cprune_mx4_dequantize(block.codes, block.scales, 40).double().t()
    loss = ((y - target.double()) ** 2).mean()
    grads = torch.autograd.grad(loss, (w64, b64, x64))
    loss = loss.detach()
    bar = 2e-5 if dtype == torch.float32 else 2e-2
    assert abs(float(error) - float(loss)) <= (1e-5 if dtype == torch.float32 else 1e-2) * float(loss)
    for got, want in zip((dweight, dbias, dx), grads):
        assert float((got.double() - want).norm()) <= bar * float(want.norm())


def test_tuning_lowers_the_error():
    errors, us = pointwise.run(c_in=48, c_out=64, keep=45, hw=7, batch=4, steps=30, groups=6)
    assert 0 < errors[-1] < 0.98 * errors[0] and us > 0
