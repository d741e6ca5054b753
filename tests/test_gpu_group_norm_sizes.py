"""Group norm and its gradient on the most pixels that a tensor may have."""
import pytest
import torch

from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def test_the_most_pixels():
    """2^31 - 1 pixels of a channel: the last superrow of eight lacks one.  Means and sums in 64 bits over parts of 2^26."""
    p, step, eps = 2 ** 31 - 1, 2 ** 26, float(torch.tensor(1e-5))
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1 << 20, generator=g, device="cuda").half().repeat(2048)[:p].reshape(1, p, 1)
    dy = torch.randn((1 << 20) + 64, generator=g, device="cuda").half().repeat(2048)[:p].reshape(1, p, 1)
    weight, bias = torch.tensor([1.5], device="cuda"), torch.tensor([0.25], device="cuda")
    y, mean, rstd = B.cprune_group_norm_act(x, 1, weight, bias, act=B.ACT_NONE, want_stats=True)
    dx, dweight, dbias = B.cprune_group_norm_act_backward(dy, x, mean, rstd, 1, weight, bias)
    parts = [slice(i, min(i + step, p)) for i in range(0, p, step)]
    total = sum(x[0, s].double().sum() for s in parts)
    squares = sum(x[0, s].double().square().sum() for s in parts)
    m64 = total / p
    r64 = (squares / p - m64 * m64 + eps) ** -0.5
    assert abs(float(mean) - m64) <= 32 * E * 6 and abs(float(rstd) - r64) <= 64 * E
    m, r = mean.double(), rstd.double()
    sums = [torch.zeros((), dtype=torch.float64, device="cuda") for _ in range(4)]
    for s in parts:
        d, xhat = dy[0, s].double(), (x[0, s].double() - m) * r
        for acc, v in zip(sums, (d, d * xhat, d.abs(), (d * xhat).abs())):
            acc += v.sum()
    assert abs(float(dbias) - sums[0]) <= 64 * E * sums[2] and abs(float(dweight) - sums[1]) <= 64 * E * 3 * sums[3]
    t1, t2 = 1.5 * sums[0] / p, 1.5 * sums[1] / p
    for s in parts:
        xhat = (x[0, s].double() - m) * r
        want = 1.5 * xhat + 0.25
        assert bool(((y[0, s].double() - want).abs() <= 2.0 ** -11 * want.abs() + 1e-5).all())
        want = r * (1.5 * dy[0, s].double() - t1 - xhat * t2)
        assert bool(((dx[0, s].double() - want).abs() <= 2.0 ** -11 * want.abs() + 1e-5).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,p,c,groups,stride", [(2 ** 22, 1, 3, 1, 4), (2 ** 21, 2, 3, 3, 4)])
def test_many_images_of_the_first_channels(n, p, c, groups, stride, dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(n, p, stride, generator=g, device="cuda").to(dtype)[..., :c] for _ in range(2))
    y, mean, rstd = B.cprune_group_norm_act(x, groups, eps=1.0, want_stats=True)
    dx, dweight, dbias = B.cprune_group_norm_act_backward(dy, x, mean, rstd, groups)
    x64, d = x.double().reshape(n, p, groups, -1), dy.double().reshape(n, p, groups, -1)
    m64 = x64.mean(dim=(1, 3), keepdim=True)
    r64 = ((x64 - m64).square().mean(dim=(1, 3), keepdim=True) + 1.0) ** -0.5
    xhat = (x64 - m64) * r64
    u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    # (groups of two or three numbers, eps 1: every term is of order one, and some 32 roundings of them)
    for got, want in ((mean, m64), (rstd, r64), (y, xhat), (dx, r64 * (d - d.mean(dim=(1, 3), keepdim=True) - xhat * (d * xhat).mean(dim=(1, 3), keepdim=True)))):
        want = want.reshape(got.shape)
        slack = 32 * E * (1 + x64.abs().amax()) * (1 + d.abs().amax())
        assert bool(((got.double() - want).abs() <= (u if got.dtype == dtype else E) * want.abs() + slack).all())
    for got, v in ((dbias, d), (dweight, d * xhat)):
        v = v.reshape(n * p, c)
        assert bool(((got.double() - v.sum(dim=0)).abs() <= 64 * E * (1 + v.abs()).sum(dim=0)).all())
