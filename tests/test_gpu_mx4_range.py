"""4-bit products at the ends of the scales, and few rows that begin at any element.

A row's blocks all have one scale here, so a result is a whole number of quarters times a power of two: the sum of at most 6500 terms of up to 36 is exact in
fp32 wherever it is a normal number.  Below 2^-126 each matrix instruction, join and output may round to a multiple of 2^-149: (k / 128 + 16) of those.
Past the largest number a sum of positive terms is an infinity."""
import math

import pytest
import torch

from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu

TABLE = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
ENDS = [0, 1, 2, 30, 64, 100, 126, 127, 128, 150, 190, 220, 252, 253, 254]


def side(rows, blocks, seed, positive, ends):
    """-> codes, scales (row r's all ends[r % 15]), the codes' values and the rows' exponents in 64 bits"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    four = torch.randint(0, 8 if positive else 16, (rows, 32 * blocks), generator=g, device="cuda", dtype=torch.uint8)
    scale = torch.tensor(ends, device="cuda")[torch.arange(rows, device="cuda") % len(ends)]
    codes = (four[:, 0::2] | four[:, 1::2] << 4).contiguous()
    v = torch.where(four > 7, -1.0, 1.0).double() * torch.tensor(TABLE, dtype=torch.float64, device="cuda")[(four & 7).int()]
    return codes, scale.to(torch.uint8)[:, None].expand(rows, blocks).contiguous(), v, scale.double() - 127


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("rows,k,c_out", [(3, 128, 47), (16, 4096, 64), (30, 1280, 100), (45, 96, 75), (60, 6400, 2000), (150, 640, 96), (500, 256, 300), (700, 2048, 1500)])
def test_products_at_the_ends_of_the_scales(rows, k, c_out, positive):
    xc, xs, xv, xe = side(rows, k // 32, 1, positive, ENDS[::-1])
    wc, ws, wv, we = side(c_out, k // 32, 2, positive, ENDS)
    sums = xv @ wv.t().contiguous()
    size = xv.abs() @ wv.abs().t().contiguous()
    power = torch.exp2(xe[:, None] + we[None])
    want, size = sums * power, size * power
    for dtype in (torch.float32, torch.bfloat16):
        y = B.cprune_mx4_matmul(xc, xs, wc, ws, B.DTYPE_OF_TORCH[dtype])
        top = torch.finfo(dtype).max
        inside = size < top * (1 - 2.0 ** -9)
        u = 0.0 if dtype == torch.float32 else 2.0 ** -8
        tiny = (k / 128 + 16) * 2.0 ** -149 * (want.abs() < 2.0 ** -126) + (0.0 if dtype == torch.float32 else 2.0 ** -133)
        bad = inside & ~((y.double() - want).abs() <= u * want.abs() + tiny)
        assert not bad.any(), (int(bad.sum()), [(ENDS[-1 - int(r) % 15], ENDS[int(o) % 15], float(y[r, o]), float(want[r, o])) for r, o in bad.nonzero()[:6]])
        if positive:
            past = want > top * (1 + 2.0 ** -8)
            assert past.any() and torch.isinf(y[past]).all() and (y[past] > 0).all()


@pytest.mark.parametrize("rows,k,c_out", [(3, 100, 40), (16, 4100, 50), (60, 333, 70), (400, 700, 300)])
def test_numbers_at_the_ends_of_their_type(rows, k, c_out):
    """Numbers of 2^-149 to 3e38 become codes within the call as they do by themselves."""
    g = torch.Generator(device="cuda").manual_seed(3)
    exponent = torch.randint(-149, 128, (rows, 1), generator=g, device="cuda")
    x = torch.ldexp(torch.rand(rows, k, generator=g, device="cuda").double() + 0.5, exponent - 1).float()
    w = torch.randn(c_out, k, generator=g, device="cuda") * 2.0 ** -10
    wc, ws = B.cprune_mx4_quantize(w)
    xc, xs = B.cprune_mx4_quantize(x)
    assert torch.isfinite(x).all() and not (xs == 255).any()
    xv, wv = (B.cprune_mx4_dequantize(c, s, k).double() for c, s in ((xc, xs), (wc, ws)))
    y = B.cprune_mx4_linear(x, wc, ws).double()
    want, size = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    bound = (k / 128 + 16) * (2.0 ** -24 * size + 2.0 ** -149)
    assert bool(((y - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("wide", [1, 13, 16])
@pytest.mark.parametrize("rows,k", [(4, 8190), (14, 4096), (16, 4097), (16, 2050), (30, 2049), (1, 33000)])
def test_few_rows_that_begin_anywhere(rows, k, wide, dtype):
    """Rows of even and odd lengths at even and odd distances give the results of the same rows without gaps."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(rows, k + wide, generator=g, device="cuda").to(dtype)[:, :k]
    wc, ws = B.cprune_mx4_quantize(torch.randn(50, k, generator=g, device="cuda") / math.sqrt(k))
    xc, xs = B.cprune_mx4_quantize(x)
    y = B.cprune_mx4_linear(x, wc, ws)
    want = B.cprune_mx4_matmul(xc, xs, wc, ws, B.DTYPE_OF_TORCH[dtype])
    assert torch.equal(xc, B.cprune_mx4_quantize(x.contiguous())[0])
    assert torch.equal(y, B.cprune_mx4_linear(x.contiguous(), wc, ws)) and torch.equal(y, want)
