"""Microscaled 4-bit codes and products on them, against the definition in 64 bits.

Codes and the numbers they stand for are exact: no tolerance.  Products: each of the k terms is exact, their sum is held in fp32: at most one rounding
of 2^-24 a matrix instruction of 128 terms, one for each join of partial sums and one for the bias, of no more than the sum of the magnitudes;
(k / 128 + 16) 2^-24 of that sum, and the type's half unit in the last place.  SiLU moves no further than 1.1 times its argument, its own roundings are
8 2^-24 (1 + |z|) of it."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def encode(x):
    """[rows, k] numbers -> (codes, scales) by the definition, in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    blocks = -(-k // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :k] = x
    v = v.reshape(rows, blocks, 32)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(v).all(axis=2)
        v = np.where(bad[..., None], 0.0, v)
        top = np.abs(v).max(axis=2)
        s = np.where(top > 0, np.maximum(0, np.frexp(top)[1] - 1 + 125), 0)
        a = np.abs(np.ldexp(v, (127 - s)[..., None]))
    dist = np.abs(a[..., None] - GRID)
    best = dist.min(axis=-1, keepdims=True)
    tied = dist == best                                  # ties to the even index
    index = np.where(tied.sum(-1) > 1, np.where(tied, np.arange(8) % 2 == 0, False).argmax(-1), tied.argmax(-1))
    four = (index + 8 * np.signbit(v)).astype(np.uint8)
    four[bad] = 0
    four = four.reshape(rows, -1)
    return four[:, 0::2] | (four[:, 1::2] << 4), np.where(bad, 255, s).astype(np.uint8)


def decode(codes, scales, k):
    four = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    v = np.where(four & 8, -1.0, 1.0) * GRID[four & 7]
    p = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v * np.repeat(p, 32, axis=1))[:, :k]


def numbers(rows, k, dtype, seed=0, wide=0):
    g = torch.Generator().manual_seed(seed + 7 * k + rows)
    x = torch.randn(rows, k + wide, generator=g) * torch.exp(1.5 * torch.randn(rows, 1, generator=g))
    return x.to(dtype).cuda()[:, :k]


def np64(t):
    return t.detach().cpu().double().numpy()


def codes_check(x):
    codes, scales = B.cprune_mx4_quantize(x)
    want_c, want_s = encode(np64(x.reshape(-1, x.shape[-1])))
    assert np.array_equal(scales.cpu().numpy(), want_s)
    got = codes.cpu().numpy()
    # (a zero's sign is kept where the block is finite)
    assert np.array_equal(got, want_c), np.argwhere(got != want_c)[:4]
    return codes, scales


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (49, 320), (7, 100), (1, 8192), (300, 83), (1025, 144), (17, 2049), (4096, 8), (2, 5)])
def test_codes(rows, k, dtype):
    x = numbers(rows, k, dtype)
    codes, scales = codes_check(x)
    for out in TYPES:
        back = B.cprune_mx4_dequantize(codes, scales, k, B.DTYPE_OF_TORCH[out])
        want = torch.from_numpy(decode(codes.cpu().numpy(), scales.cpu().numpy(), k)).to(out)
        assert torch.equal(back.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wide", [1, 8, 13])
def test_codes_of_the_first_numbers_of_wider_rows(wide, dtype):
    for k in (5, 32, 77, 144):
        codes_check(numbers(33, k, dtype, wide=wide))


def test_every_16_bit_number_and_every_tie():
    for dtype in (torch.float16, torch.bfloat16):
        every = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dtype)
        every = every[torch.isfinite(every.float())]
        x = torch.zeros(every.numel(), 32, dtype=dtype)
        x[:, 3] = every                                 # each as its block's largest
        codes_check(x.cuda())
        x = every[: every.numel() // 32 * 32].reshape(-1, 32)       # and among its neighbours
        codes_check(x.cuda().contiguous())
    ties = torch.tensor([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.99, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -7, -0.0, 0.2500001, 0.2499999, 2.5000002,
                         4.9999995, 4, 3, 2, 1.5, 1, 0.5, 1e-30, -1e-30])
    ties[8] = 4.5       # (the largest is 7.99: the scale is 1)
    exponents = [-149, -148, -140, -130, -127, -126, -125, -124, -100, -1, 0, 1, 60, 124, 125]
    x = torch.stack([torch.ldexp(ties.double(), torch.tensor(e)).float() for e in exponents])
    codes_check(x.cuda())


def test_blocks_with_infinity_or_nan_and_the_ends_of_the_scales():
    x = torch.randn(6, 100, generator=torch.Generator().manual_seed(1))
    x[0, 5], x[1, 40], x[2, 99], x[3, 64:96] = math.inf, -math.inf, math.nan, 0
    x[4, :32], x[5, :32] = 3.4e38, 2.0 ** -149
    codes, scales = codes_check(x.cuda())
    back = B.cprune_mx4_dequantize(codes, scales, 100)
    bad = torch.zeros(6, 100, dtype=torch.bool)
    bad[0, :32], bad[1, 32:64], bad[2, 96:] = True, True, True
    assert torch.equal(torch.isnan(back.cpu()), bad)
    # any byte as a scale, any code
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).reshape(256, 16, 16).transpose(1, 2).reshape(256, 256).contiguous().cuda()
    scales = torch.arange(256, dtype=torch.uint8).reshape(256, 1).repeat(1, 16).contiguous().cuda()
    for out in TYPES:
        back = B.cprune_mx4_dequantize(codes, scales, 512, B.DTYPE_OF_TORCH[out]).cpu()
        want = torch.from_numpy(decode(codes.cpu().numpy(), scales.cpu().numpy(), 512)).to(out)
        assert torch.equal(torch.isnan(back), torch.isnan(want)) and torch.equal(back.nan_to_num(0.0), want.nan_to_num(0.0))


def act64(z, act):
    if act == B.ACT_SILU:
        with np.errstate(over="ignore"):
            return z / (1 + np.exp(-z))
    return np.clip(z, -np.inf if act == B.ACT_NONE else 0, 6 if act == B.ACT_RELU6 else np.inf)


def product_check(y, xv, wv, bias, act, dtype):
    k = xv.shape[1]
    z = xv @ wv.T
    size = np.abs(xv) @ np.abs(wv).T
    if bias is not None:
        z, size = z + np64(bias), size + np.abs(np64(bias))
    want = act64(z, act)
    slack = (k / 128 + 16) * E24 * size * (1.1 if act == B.ACT_SILU else 1)
    if act == B.ACT_SILU:
        slack = slack + 8 * E24 * (1 + np.abs(z)) * np.abs(want)
    got = np64(y)
    if dtype == torch.float16:      # past its largest number, a result is an infinity
        past = np.isinf(got) & (np.abs(want) >= 65520 - slack) & (np.sign(got) == np.sign(want))
        got = np.where(past, want, got)
    over = np.abs(got - want) - (U[dtype] * np.abs(want) + slack + TINY[dtype])
    assert over.max() <= 0, f"{np.count_nonzero(over > 0)} of {over.size} past the bound"


E24 = 2.0 ** -24
# rows, k, c_out: one of each, tails of every tile, few rows of long sums, many rows of short ones, both large
PRODUCTS = [(1, 1, 1), (1, 32, 16), (1, 4096, 1000), (3, 70, 5), (16, 128, 64), (17, 129, 65), (33, 31, 33), (32, 1280, 1000), (5, 8192, 48), (64, 640, 129),
            (100, 333, 77), (129, 1000, 257), (255, 96, 31), (512, 512, 512), (513, 544, 300), (1000, 36, 24), (2049, 160, 100), (4000, 100, 3), (300, 4100, 520),
            (1024, 2048, 768), (8, 2000, 4100), (2, 20000, 40), (64, 700, 70), (70, 1300, 130), (90, 5000, 33),
            (1100, 1100, 1300), (2100, 130, 2200), (3000, 4100, 3100), (40, 600, 1000), (1500, 640, 90), (33, 8, 4097)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,c_out", PRODUCTS)
def test_products(rows, k, c_out, dtype):
    x, w = numbers(rows, k, dtype), numbers(c_out, k, torch.float32, seed=1) / math.sqrt(k)
    bias = numbers(1, c_out, torch.float32, seed=2)[0].contiguous()
    wc, ws = B.cprune_mx4_quantize(w)
    wv = decode(*encode(np64(w)), k)
    xv = decode(*encode(np64(x)), k)
    for act, b in ((B.ACT_NONE, None), (B.ACT_SILU, bias), (B.ACT_RELU6, bias)):
        y = B.cprune_mx4_linear(x, wc, ws, b, act)
        product_check(y, xv, wv, b, act, dtype)
        assert torch.equal(y, B.cprune_mx4_linear(x, wc, ws, b, act))
    xc, xs = B.cprune_mx4_quantize(x)
    y = B.cprune_mx4_matmul(xc, xs, wc, ws, B.DTYPE_OF_TORCH[dtype], bias, B.ACT_RELU)
    product_check(y, xv, wv, bias, B.ACT_RELU, dtype)


@pytest.mark.parametrize("wide", [1, 8, 13])
def test_products_of_the_first_numbers_of_wider_rows(wide):
    for dtype in TYPES:
        for rows, k, c_out in [(1, 77, 40), (50, 144, 96), (400, 130, 200)]:
            x, w = numbers(rows, k, dtype, wide=wide), numbers(c_out, k, torch.float32, seed=1)
            wc, ws = B.cprune_mx4_quantize(w)
            y = B.cprune_mx4_linear(x, wc, ws)
            product_check(y, decode(*encode(np64(x)), k), decode(*encode(np64(w)), k), None, B.ACT_NONE, dtype)


def test_an_infinity_spoils_its_own_row_or_column_only():
    for rows in (1, 40, 700):
        x, w = numbers(rows, 200, torch.bfloat16), numbers(150, 200, torch.float32, seed=1)
        wc, ws = B.cprune_mx4_quantize(w)
        clean = B.cprune_mx4_linear(x, wc, ws, act=B.ACT_RELU)
        x[rows // 2, 33] = math.inf
        y = B.cprune_mx4_linear(x, wc, ws, act=B.ACT_RELU)
        keep = torch.arange(rows, device="cuda") != rows // 2
        assert torch.isnan(y[rows // 2]).all() and torch.equal(y[keep], clean[keep])
        w[7, 199] = math.nan
        wc, ws = B.cprune_mx4_quantize(w)
        y = B.cprune_mx4_linear(x, wc, ws, act=B.ACT_RELU)
        col = torch.arange(150, device="cuda") != 7
        assert torch.isnan(y[:, 7]).all() and torch.equal(y[keep][:, col], clean[keep][:, col])


def test_leading_sizes_and_outputs_that_hold_nothing_else():
    x, w = numbers(24, 64, torch.float16), numbers(40, 64, torch.float32, seed=1)
    wc, ws = B.cprune_mx4_quantize(w)
    y = B.cprune_mx4_linear(x.reshape(2, 3, 4, 64), wc, ws)
    assert y.shape == (2, 3, 4, 40) and torch.equal(y.reshape(24, 40), B.cprune_mx4_linear(x, wc, ws))
    xc, xs = B.cprune_mx4_quantize(x)
    for rows, c_out in ((24, 40), (23, 39), (1, 37)):
        for off in (0, 1, 3):
            out = torch.full((rows * c_out + 128,), 9.0, dtype=torch.float16, device="cuda")
            st = B.lib().cprune_mx4_matmul(xc.data_ptr(), xs.data_ptr(), rows, 64, wc.data_ptr(), ws.data_ptr(), c_out, None, 0, B.F16,
                                           out.data_ptr() + 2 * (64 + off), None, 0, torch.cuda.current_stream().cuda_stream)
            assert st == B.OK
            assert torch.equal(out[64 + off:64 + off + rows * c_out].reshape(rows, c_out), y.reshape(24, 40)[:rows, :c_out])
            assert (out[:64 + off] == 9).all() and (out[64 + off + rows * c_out:] == 9).all()


def test_on_another_stream_and_in_a_graph():
    x, w = numbers(50, 320, torch.bfloat16), numbers(96, 320, torch.float32, seed=1)
    wc, ws = B.cprune_mx4_quantize(w)
    y = B.cprune_mx4_linear(x, wc, ws, act=B.ACT_SILU)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = B.cprune_mx4_linear(x, wc, ws, act=B.ACT_SILU, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, y)
    xs = x.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys = B.cprune_mx4_linear(xs, wc, ws, act=B.ACT_SILU)
        back = B.cprune_mx4_dequantize(*B.cprune_mx4_quantize(xs), 320, B.BF16)
    for i in range(4):
        xs.copy_(x * (i - 1.5))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys, B.cprune_mx4_linear(xs, wc, ws, act=B.ACT_SILU))
        assert torch.equal(back, B.cprune_mx4_dequantize(*B.cprune_mx4_quantize(xs), 320, B.BF16))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,c_out", [(14, 6145, 33), (4, 8193, 70), (16, 2049, 9), (1, 40001, 20)])
def test_few_rows_of_long_and_odd_sums(rows, k, c_out, dtype):
    x, w = numbers(rows, k, dtype), numbers(c_out, k, torch.float32, seed=1) / math.sqrt(k)
    wc, ws = B.cprune_mx4_quantize(w)
    y = B.cprune_mx4_linear(x, wc, ws)
    product_check(y, decode(*encode(np64(x)), k), decode(*encode(np64(w)), k), None, B.ACT_NONE, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,c_out", [(8200, 4100, 8000), (1300, 700, 2000), (2050, 70, 2500), (700, 5000, 600)])
def test_products_of_many_tiles(rows, k, c_out, dtype):
    """Tiles of every width, all outputs against a product in 64 bits."""
    def codes_of(n, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        blocks = -(-k // 32)
        codes = torch.randint(0, 256, (n, blocks * 16), generator=g, device="cuda", dtype=torch.uint8)
        scales = torch.randint(120, 126, (n, blocks), generator=g, device="cuda", dtype=torch.uint8)
        four = torch.stack([codes & 15, codes >> 4], dim=2).reshape(n, -1)
        four[:, k:] = 0
        packed = (four[:, 0::2] | four[:, 1::2] << 4).contiguous()
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        v = torch.where(four > 7, -1.0, 1.0).double() * table[(four & 7).int()] * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)
        return packed, scales, v[:, :k].contiguous()
    xc, xs, xv = codes_of(rows, 1)
    wc, ws, wv = codes_of(c_out, 2)
    bias = torch.randn(c_out, generator=torch.Generator().manual_seed(3)).cuda()
    y = B.cprune_mx4_matmul(xc, xs, wc, ws, B.DTYPE_OF_TORCH[dtype], bias).double()
    wt = wv.t().contiguous()
    want, size = xv @ wt + bias.double(), xv.abs() @ wt.abs() + bias.double().abs()
    over = (y - want).abs() - (U[dtype] * want.abs() + (k / 128 + 16) * E24 * size + TINY[dtype])
    assert over.max().item() <= 0, f"{int((over > 0).sum())} of {over.numel()} past the bound"
