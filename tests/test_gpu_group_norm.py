"""Group norm with its activation, channels last, and its gradient, against the formula in 64 bits.

Bounds.  u is the type's half unit in the last place (2^-24, 2^-11, 2^-8), e = 2^-24.  Forward: x - mean loses e (|x| + |mean|), the statistics and the few
products and sums behind them a few e of what they hold, the sigmoid a few e more and its exponential e |z|: 32 e of the sum of the magnitudes
covers them with a factor of about four.  Backward: the same on each term of dx, the two means relative to the means of the terms' magnitudes; sums
over many numbers are chains of at most a few hundred additions joined in 64 bits, whose errors add up like their square root: 64 e of the
magnitudes' sum.  Clamps: dy is 0 where z lies within 1e-4 of a kink, so that both sides take the same branch."""
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
E = 2.0 ** -24
EPS = 1e-5

# (n, h, w, c, groups): one pixel, one channel, pixels that do not fill a superrow, odd and prime channel counts, groups of one and of all, one image of
# many pixels, many images, channel counts past a work-group's vectors
SHAPES = [(1, 1, 1, 1, 1), (3, 1, 1, 8, 2), (2, 1, 5, 3, 1), (1, 7, 7, 1, 1), (2, 3, 3, 83, 1), (2, 5, 7, 83, 83), (1, 14, 14, 96, 8), (4, 9, 11, 30, 5),
          (2, 28, 28, 64, 32), (1, 56, 57, 24, 24), (3, 4, 4, 1280, 32), (2, 3, 5, 2051, 7), (130, 2, 2, 16, 4), (1, 112, 112, 16, 2), (1, 1, 3, 5000, 8),
          (1, 1, 2, 4096, 1), (1, 211, 97, 2, 1), (5, 17, 13, 45, 9), (2, 64, 64, 40, 4)]


def make(shape, dtype, wide, seed=0, mean=0.5):
    n, h, w, c, _ = shape
    g = torch.Generator().manual_seed(seed + 31 * c + h)
    x = torch.randn(n, h, w, c + wide, generator=g) * (0.5 + torch.rand(c + wide, generator=g)) + mean * torch.randn(c + wide, generator=g)
    dy = torch.randn(n, h, w, c + wide, generator=g)
    weight = 0.5 + torch.rand(c, generator=g)
    bias = 0.3 * torch.randn(c, generator=g)
    return x.to(dtype).cuda()[..., :c], dy.to(dtype).cuda()[..., :c], weight.cuda(), bias.cuda()


def act64(z, act):
    if act == B.ACT_SILU:
        return z / (1 + np.exp(-z))
    return np.clip(z, -np.inf if act == B.ACT_NONE else 0, 6 if act == B.ACT_RELU6 else np.inf)


def slope64(z, act):
    if act == B.ACT_SILU:
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    lo, hi = (-np.inf if act == B.ACT_NONE else 0), (6 if act == B.ACT_RELU6 else np.inf)
    return ((z > lo) & (z < hi)).astype(np.float64)


def wide64(t):
    return t.detach().cpu().double().numpy()


def check(got, want, bound, what):
    got = wide64(got)
    assert got.shape == want.shape, what
    over = np.abs(got - want) - bound
    assert not np.isnan(got).any(), what
    assert over.max() <= 0, f"{what}: {np.count_nonzero(over > 0)} of {over.size} past the bound, worst {np.max(np.abs(got - want) / bound):.2f} of it"


def stats64(x, groups):
    n, c = x.shape[0], x.shape[-1]
    v = x.reshape(n, -1, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1 / np.sqrt(var + np.float64(np.float32(EPS)))


def spread(s, shape):
    """[n, groups] -> over [n, h, w, c]"""
    n, h, w, c, groups = shape
    return np.repeat(s, c // groups, axis=1).reshape(n, 1, 1, c)


def forward_check(shape, dtype, wide, act, affine, mean=0.5):
    x, _, weight, bias = make(shape, dtype, wide, mean=mean)
    y, m, r = B.cprune_group_norm_act(x, shape[4], weight if affine else None, bias if affine else None, eps=EPS, act=act, want_stats=True)
    again = B.cprune_group_norm_act(x, shape[4], weight if affine else None, bias if affine else None, eps=EPS, act=act)
    assert torch.equal(y, again)
    x64 = wide64(x)
    w64, b64 = (wide64(weight), wide64(bias)) if affine else (1.0, 0.0)
    mean64, rstd64 = stats64(x64, shape[4])
    top = np.abs(x64).reshape(shape[0], -1, shape[4], shape[3] // shape[4]).max(axis=(1, 3))
    check(m, mean64, 32 * E * top, f"mean {shape}")
    check(r, rstd64, 32 * E * rstd64 * (1 + rstd64 * np.abs(mean64)), f"rstd {shape}")
    mm, rr, tt = spread(mean64, shape), spread(rstd64, shape), spread(top, shape)
    z = (x64 - mm) * rr * w64 + b64
    want = act64(z, act)
    size = (np.abs(x64) + tt) * rr * np.abs(w64) + np.abs(b64)
    slack = 32 * E * size * (1 + rr * np.abs(mm)) * (1 + np.abs(z) * (act == B.ACT_SILU))
    check(y, want, U[dtype] * np.abs(want) + slack + TINY[dtype], f"y {shape} {dtype} act {act}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    forward_check(shape, dtype, 0, B.ACT_SILU, True)
    forward_check(shape, dtype, 0, B.ACT_NONE, False)


@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_RELU6, B.ACT_SILU])
@pytest.mark.parametrize("wide", [1, 4, 8, 13])
def test_forward_of_the_first_channels_of_a_wider_map(wide, act):
    for dtype in TYPES:
        for shape in [(2, 9, 7, 45, 5), (3, 14, 14, 64, 8), (1, 5, 3, 12, 1)]:
            forward_check(shape, dtype, wide, act, True)


def test_forward_of_numbers_far_from_zero():
    """A mean a thousand spreads away: differences of large sums would leave nothing of the variance."""
    forward_check((2, 40, 31, 48, 6), torch.float32, 0, B.ACT_NONE, True, mean=1000.0)
    # a border of zeros around such numbers
    x = torch.full((1, 30, 30, 8), 500.0, device="cuda") + torch.randn(1, 30, 30, 8, generator=torch.Generator().manual_seed(3)).cuda()
    x[:, 0], x[:, :, 0] = 0, 0
    y, m, r = B.cprune_group_norm_act(x, 8, want_stats=True)
    mean64, rstd64 = stats64(wide64(x), 8)
    check(r, rstd64, 32 * E * rstd64 * (1 + rstd64 * np.abs(mean64)), "rstd")


def backward_check(shape, dtype, wide, act, affine):
    x, dy, weight, bias = make(shape, dtype, wide, seed=9)
    groups = shape[4]
    x64 = wide64(x)
    mean64, rstd64 = stats64(x64, groups)
    mean, rstd = torch.from_numpy(mean64).float().cuda(), torch.from_numpy(rstd64).float().cuda()
    mm, rr = spread(wide64(mean), shape), spread(wide64(rstd), shape)
    w64, b64 = (wide64(weight), wide64(bias)) if affine else (np.ones(shape[3]), np.zeros(shape[3]))
    xhat = (x64 - mm) * rr
    z = xhat * w64 + b64
    if act in (B.ACT_RELU, B.ACT_RELU6):
        near = (np.abs(z) < 1e-4) | ((np.abs(z - 6) < 1e-4) if act == B.ACT_RELU6 else False)
        dy[torch.from_numpy(near).cuda()] = 0
    dz = wide64(dy) * slope64(z, act)
    m = x64[0].size // groups
    per = lambda v: spread(v.reshape(shape[0], -1, groups, shape[3] // groups).sum(axis=(1, 3)) / m, shape)
    t1, t2 = per(dz * w64), per(dz * w64 * xhat)
    want = rr * (dz * w64 - t1 - xhat * t2)
    dx, dweight, dbias = B.cprune_group_norm_act_backward(dy, x, mean, rstd, groups, weight if affine else None, bias if affine else None, act=act)
    off = (np.abs(x64) + np.abs(mm)) * rr                      # what xhat may be off by, in e
    soft = 1 + (np.abs(z) + off) * (act == B.ACT_SILU)         # how that moves the slope
    a = np.abs(wide64(dy)) * np.abs(w64)
    size = a * soft + per(a * soft) + np.abs(xhat) * per(a * soft * (np.abs(xhat) + off)) + off * np.abs(t2)
    check(dx, want, U[dtype] * np.abs(want) + 64 * E * rr * size + TINY[dtype], f"dx {shape} {dtype} act {act}")
    d = np.abs(wide64(dy)) * soft
    check(dbias, dz.sum(axis=(0, 1, 2)), 64 * E * d.sum(axis=(0, 1, 2)) + 1e-30, f"dbias {shape}")
    check(dweight, (dz * xhat).sum(axis=(0, 1, 2)), 64 * E * (d * (np.abs(xhat) + off)).sum(axis=(0, 1, 2)) + 1e-30, f"dweight {shape}")
    twice = B.cprune_group_norm_act_backward(dy, x, mean, rstd, groups, weight if affine else None, bias if affine else None, act=act)
    assert all(torch.equal(p, q) for p, q in zip((dx, dweight, dbias), twice))
    alone = B.cprune_group_norm_act_backward(dy, x, mean, rstd, groups, weight if affine else None, bias if affine else None, act=act,
                                             want_vectors=False)
    assert torch.equal(alone[0], dx) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype):
    backward_check(shape, dtype, 0, B.ACT_SILU, True)
    backward_check(shape, dtype, 0, B.ACT_RELU, False)


@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU, B.ACT_RELU6, B.ACT_SILU])
@pytest.mark.parametrize("wide", [1, 4, 8, 13])
def test_backward_of_the_first_channels_of_a_wider_map(wide, act):
    for dtype in TYPES:
        for shape in [(2, 9, 7, 45, 5), (3, 14, 14, 64, 8), (1, 5, 3, 12, 1)]:
            backward_check(shape, dtype, wide, act, True)


def test_backward_with_a_dense_gradient_of_a_slice():
    x, _, weight, bias = make((2, 6, 5, 24, 3), torch.bfloat16, 8)
    dy = torch.randn(2, 6, 5, 24, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    _, mean, rstd = B.cprune_group_norm_act(x, 3, weight, bias, act=B.ACT_SILU, want_stats=True)
    a = B.cprune_group_norm_act_backward(dy, x, mean, rstd, 3, weight, bias, act=B.ACT_SILU)
    b = B.cprune_group_norm_act_backward(dy, x.contiguous(), mean, rstd, 3, weight, bias, act=B.ACT_SILU)
    for p, q in zip(a, b):      # (another order of the sums)
        assert torch.allclose(p.float(), q.float(), rtol=2.0 ** -7, atol=1e-5)


@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_SILU])
def test_gradient_against_differences(act):
    """<gradient, direction> against the difference of sum(y dy) at both ends of a short step: the step's square (1e-4, times the third derivative, of
    order one) and the outputs' rounding (2^-24 a number, random, over 2 h = 0.02) stay below 1e-3 of the gradients' and directions' lengths."""
    shape = (3, 6, 7, 20, 4)
    x, dy, weight, bias = make(shape, torch.float32, 0, seed=4)
    g = torch.Generator().manual_seed(5)
    h = 1e-2

    def loss(x, weight, bias):
        return float((B.cprune_group_norm_act(x, 4, weight, bias, act=act).double() * dy.double()).sum())

    _, mean, rstd = B.cprune_group_norm_act(x, 4, weight, bias, act=act, want_stats=True)
    grads = B.cprune_group_norm_act_backward(dy, x, mean, rstd, 4, weight, bias, act=act)
    at = [x, weight, bias]
    for i, grad in enumerate(grads):
        v = torch.randn(at[i].shape, generator=g).cuda()
        ends = []
        for sign in (1, -1):
            moved = list(at)
            moved[i] = at[i] + sign * h * v
            ends.append(loss(*moved))
        slope = (ends[0] - ends[1]) / (2 * h)
        along = float((grad.double() * v.double()).sum())
        assert abs(slope - along) <= 1e-3 * float(grad.double().norm() * v.double().norm()), (i, slope, along)


def test_infinity_and_nan_stay_in_their_image_and_group():
    for bad in (math.inf, -math.inf, math.nan):
        for dtype in TYPES:
            x, dy, weight, bias = make((3, 5, 5, 24, 4), dtype, 0)
            clean, mean, rstd = B.cprune_group_norm_act(x, 4, weight, bias, act=B.ACT_RELU, want_stats=True)
            x[1, 2, 3, 8] = bad
            y = B.cprune_group_norm_act(x, 4, weight, bias, act=B.ACT_RELU)
            spoilt = torch.zeros_like(y, dtype=torch.bool)
            spoilt[1, :, :, 6:12] = True
            assert torch.isnan(y[spoilt]).all() and torch.equal(y[~spoilt], clean[~spoilt])


def test_equal_numbers_have_no_spread():
    x = torch.full((2, 4, 4, 16), 3.0, device="cuda", dtype=torch.float16)
    bias = torch.linspace(-1, 1, 16, device="cuda")
    y, mean, rstd = B.cprune_group_norm_act(x, 4, None, bias, eps=1e-5, want_stats=True)
    assert torch.equal(y, bias.half().expand_as(y)) and torch.all(mean == 3)
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)


def test_nothing_outside_is_written_and_addresses_need_no_alignment():
    shape, pad = (2, 5, 3, 83, 1), 64
    count = math.prod(shape[:4])
    for dtype in TYPES:
        x, _, weight, bias = make(shape, dtype, 0)
        want = B.cprune_group_norm_act(x, 1, weight, bias)
        d = B.NormDesc(2, 15, 83, 1, B.DTYPE_OF_TORCH[dtype], 0, 83, 83, 1e-5)
        ws = torch.empty(B.lib().cprune_group_norm_workspace_bytes(C.byref(d), 0), dtype=torch.uint8, device="cuda")
        for off in (0, 1, 3):
            xin = torch.zeros(count + 2 * pad, dtype=dtype, device="cuda")
            xin[pad + off:pad + off + count] = x.flatten()
            y = torch.full((count + 2 * pad,), 7.0, dtype=dtype, device="cuda")
            es = y.element_size()
            st = B.lib().cprune_group_norm_act(d, xin.data_ptr() + (pad + off) * es, weight.data_ptr(), bias.data_ptr(),
                                               y.data_ptr() + (pad + off) * es, None, None, ws.data_ptr(), ws.numel(),
                                               torch.cuda.current_stream().cuda_stream)
            assert st == B.OK
            assert torch.equal(y[pad + off:pad + off + count], want.flatten())
            assert (y[:pad + off] == 7).all() and (y[pad + off + count:] == 7).all()


def test_on_another_stream_and_in_a_graph():
    x, dy, weight, bias = make((2, 14, 14, 40, 4), torch.bfloat16, 0)
    y, mean, rstd = B.cprune_group_norm_act(x, 4, weight, bias, act=B.ACT_SILU, want_stats=True)
    grads = B.cprune_group_norm_act_backward(dy, x, mean, rstd, 4, weight, bias, act=B.ACT_SILU)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = B.cprune_group_norm_act(x, 4, weight, bias, act=B.ACT_SILU, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, y)

    xs = x.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys, ms, rs = B.cprune_group_norm_act(xs, 4, weight, bias, act=B.ACT_SILU, want_stats=True)
        gs = B.cprune_group_norm_act_backward(dy, xs, ms, rs, 4, weight, bias, act=B.ACT_SILU)
    for i in range(4):
        xs.copy_(x * (1 + i))
        graph.replay()
        torch.cuda.synchronize()
        y, mean, rstd = B.cprune_group_norm_act(xs, 4, weight, bias, act=B.ACT_SILU, want_stats=True)
        grads = B.cprune_group_norm_act_backward(dy, xs, mean, rstd, 4, weight, bias, act=B.ACT_SILU)
        assert torch.equal(ys, y) and all(torch.equal(p, q) for p, q in zip(gs, grads)), i


# superrows wider than a work-group, of few groups (some across two work-groups) and of many; few and large slabs; groups summed by more than a wavefront
FORMS = [(2, 20, 21, 1051, 1), (3, 9, 10, 1052, 4), (2, 30, 31, 1290, 6), (1, 33, 40, 1300, 100), (1, 5, 300, 1300, 65), (4, 4, 55, 239, 1), (2, 77, 16, 33, 11),
         (2, 15, 16, 99, 3), (2, 40, 41, 160, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", FORMS)
def test_forms(shape, dtype):
    forward_check(shape, dtype, 0, B.ACT_SILU, True)
    forward_check(shape, dtype, 5, B.ACT_RELU, False)
    backward_check(shape, dtype, 0, B.ACT_SILU, True)
    backward_check(shape, dtype, 5, B.ACT_NONE, False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(20, 67, 9, 98, 49), (31, 108, 10, 80, 4), (13, 38, 30, 160, 16)])
def test_forms_of_large_slabs(shape, dtype):
    forward_check(shape, dtype, 0, B.ACT_SILU, True)
    backward_check(shape, dtype, 0, B.ACT_SILU, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(2, 10, 109, 3, 3), (2, 9, 13, 7, 7), (3, 11, 5, 6, 3), (2, 40, 41, 9, 3), (1, 300, 301, 3, 3), (1, 200, 301, 7, 7)])
def test_vectors_that_end_in_their_first_group_again(shape, dtype):
    """Fewer channels than a vector has, or one less than it takes to come back: first and last element of one group, others between."""
    forward_check(shape, dtype, 0, B.ACT_SILU, True)
    backward_check(shape, dtype, 0, B.ACT_SILU, True)
