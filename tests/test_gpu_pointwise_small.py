"""Gradients of the pointwise block where an answer's share of the error is small."""
import numpy as np
import pytest
import torch

from paper_2207_01260_amd import binding as B
from test_gpu_pointwise import block_of

pytestmark = pytest.mark.gpu


def formula(block, x, target):
    """Error and gradients by weight, bias and x in 64 bits, the codes' rounding of the activations passed through."""
    n, h, w, c = x.shape
    x64, w64, b64 = x.double().requires_grad_(), block.weight.double().requires_grad_(), block.bias.double().requires_grad_()
    v = x64.reshape(n, h * w, block.groups, c // block.groups)
    mean, var = v.mean(dim=(1, 3), keepdim=True), v.var(dim=(1, 3), keepdim=True, correction=0)
    a = ((v - mean) / torch.sqrt(var + np.float64(np.float32(1e-5)))).reshape(x.shape) * w64 + b64
    z = a * torch.sigmoid(a)
    rounded = B.cprune_group_norm_act(x, block.groups, block.weight, block.bias, act=B.ACT_SILU)
    z = z + (B.cprune_mx4_dequantize(*B.cprune_mx4_quantize(rounded), c).double().reshape(z.shape) - z).detach()
    y = z @ B.cprune_mx4_dequantize(block.codes, block.scales, c).double().t().contiguous()
    error = ((y - target.double()) ** 2).mean()
    return error.detach(), torch.autograd.grad(error, (w64, b64, x64))


@pytest.mark.parametrize("shape", [(3, 7, 6), (4, 56, 56)])
def test_gradients_of_many_fp16_numbers(shape):
    """An answer's share of the mean error's gradient, 2 miss / count, is below fp16's normal numbers for 10^4 answers and below all of them for 10^7.  dy and dz
    are rounded to 2^-12 each, at random: an eighth of what bf16 is held to."""
    _, block, x = block_of(40, 64, 45, 5, torch.float16, shape)
    target = block.full(x) + 0.1
    error, dweight, dbias, dx = block.gradients(x, target)
    want_error, want = formula(block, x, target)
    assert abs(float(error) - float(want_error)) <= 1.25e-3 * float(want_error)
    for got, w in zip((dweight, dbias, dx), want):
        assert got.shape == w.shape and float((got.double() - w).norm()) <= 2.5e-3 * float(w.norm())
