"""What the group norm and the 4-bit calls refuse, before anything is launched; needs no GPU."""
import math

import pytest
import torch

from paper_2207_01260_amd import binding as B

FAKE = 0x1000   # never dereferenced: validation fails first


def _norm(**kw):
    d = dict(n=2, pixels=9, c=12, groups=3, dtype=B.F32, act=0, x_stride=12, dy_stride=12, eps=1e-5)
    d.update(kw)
    return B.NormDesc(*d.values())


BAD_NORMS = [dict(n=0), dict(pixels=0), dict(c=0), dict(groups=0), dict(groups=5), dict(groups=24), dict(groups=-3), dict(dtype=3), dict(dtype=-1),
             dict(act=4), dict(act=-1), dict(x_stride=11), dict(n=1 << 20, pixels=1 << 10), dict(n=3, pixels=3, x_stride=1 << 28)]


@pytest.mark.parametrize("kw", BAD_NORMS + [dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)])
def test_norm_refuses(kw):
    L, d = B.lib(), _norm(**kw)
    assert L.cprune_group_norm_act(d, FAKE, None, None, FAKE, None, None, FAKE, 1 << 40, None) == B.ERR_INVALID_ARG
    assert L.cprune_group_norm_workspace_bytes(d, 0) == 0


@pytest.mark.parametrize("kw", BAD_NORMS + [dict(dy_stride=11)])
def test_norm_gradient_refuses(kw):
    L, d = B.lib(), _norm(**kw)
    assert L.cprune_group_norm_act_backward(d, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, None, FAKE, 1 << 40, None) == B.ERR_INVALID_ARG
    assert L.cprune_group_norm_workspace_bytes(d, 1) == 0


def test_norm_refuses_missing_pointers_and_scratch():
    L, d = B.lib(), _norm(n=2, pixels=1 << 16, c=12)      # (a map that needs scratch)
    need, back = L.cprune_group_norm_workspace_bytes(d, 0), L.cprune_group_norm_workspace_bytes(d, 1)
    assert need > 0 and back > 0
    f = lambda x=FAKE, y=FAKE, ws=FAKE, size=need: L.cprune_group_norm_act(d, x, None, None, y, None, None, ws, size, None)
    assert f(x=None) == f(y=None) == B.ERR_INVALID_ARG
    assert f(ws=None) == f(size=need - 1) == B.ERR_WORKSPACE
    assert L.cprune_group_norm_act(None, FAKE, None, None, FAKE, None, None, FAKE, need, None) == B.ERR_INVALID_ARG
    g = lambda dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, ws=FAKE, size=back: L.cprune_group_norm_act_backward(
        d, dy, x, mean, rstd, None, None, dx, None, None, ws, size, None)
    assert g(dy=None) == g(x=None) == g(mean=None) == g(rstd=None) == g(dx=None) == B.ERR_INVALID_ARG
    assert g(ws=None) == g(size=back - 1) == B.ERR_WORKSPACE
    # more blocks than one launch has
    assert L.cprune_group_norm_act(_norm(n=1 << 27, pixels=1, c=1, groups=1, x_stride=1), FAKE, None, None, FAKE, None, None, FAKE, 1 << 40,
                                   None) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("args", [(0, 32, 32, 0), (4, 0, 32, 0), (4, 33, 32, 0), (4, 32, 32, 3), (4, 32, 32, -1), (1 << 20, 1, 1 << 12, 0),
                                  (1 << 26, 2, 2, 0), (-1, 32, 32, 0), (1, 0x7fffffff, 0x7fffffff, 0)])
def test_quantize_refuses(args):
    rows, k, stride, dtype = args
    L = B.lib()
    assert L.cprune_mx4_quantize(FAKE, rows, k, stride, dtype, FAKE, FAKE, None) == B.ERR_INVALID_ARG


def test_codes_refuse_missing_and_unaligned_pointers():
    L = B.lib()
    q = lambda x=FAKE, c=FAKE, s=FAKE: L.cprune_mx4_quantize(x, 4, 32, 32, 0, c, s, None)
    assert q(x=None) == q(c=None) == q(s=None) == q(c=FAKE + 8) == B.ERR_INVALID_ARG
    d = lambda c=FAKE, s=FAKE, y=FAKE, rows=4, k=32, dtype=0: L.cprune_mx4_dequantize(c, s, rows, k, dtype, y, None)
    assert d(c=None) == d(s=None) == d(y=None) == d(c=FAKE + 8) == d(rows=0) == d(k=0) == d(dtype=9) == B.ERR_INVALID_ARG


def test_products_refuse():
    L = B.lib()
    m = lambda xc=FAKE, xs=FAKE, rows=4, k=64, wc=FAKE, ws=FAKE, c_out=8, act=0, dtype=0, y=FAKE, scratch=FAKE, size=1 << 30: L.cprune_mx4_matmul(
        xc, xs, rows, k, wc, ws, c_out, None, act, dtype, y, scratch, size, None)
    for kw in (dict(xc=None), dict(xs=None), dict(wc=None), dict(ws=None), dict(y=None), dict(xc=FAKE + 4), dict(wc=FAKE + 4), dict(rows=0), dict(k=0),
               dict(c_out=0), dict(act=4), dict(act=-1), dict(dtype=3), dict(rows=1 << 26, k=1), dict(c_out=1 << 26, k=1), dict(rows=1 << 20, c_out=1 << 12)):
        assert m(**kw) == B.ERR_INVALID_ARG, kw
    big = dict(rows=4096, k=4096, c_out=4096)       # (a product that needs scratch)
    need = L.cprune_mx4_matmul_workspace_bytes(4096, 4096, 4096)
    assert need > 0 and L.cprune_mx4_matmul_workspace_bytes(4096, 0, 4096) == 0
    assert m(scratch=None, **big) == m(size=need - 1, **big) == B.ERR_WORKSPACE
    assert m(scratch=FAKE + 8, **big) == B.ERR_INVALID_ARG
    f = lambda x=FAKE, rows=4, k=64, stride=64, wc=FAKE, wsc=FAKE, c_out=8, act=0, dtype=0, y=FAKE, ws=FAKE, size=1 << 30: L.cprune_mx4_linear(
        x, rows, k, stride, wc, wsc, c_out, None, act, dtype, y, ws, size, None)
    for kw in (dict(x=None), dict(wc=None), dict(wsc=None), dict(y=None), dict(wc=FAKE + 4), dict(rows=0), dict(k=0), dict(c_out=0), dict(stride=63),
               dict(act=4), dict(dtype=3), dict(rows=1 << 26, k=1, stride=1), dict(rows=1 << 20, k=64, stride=1 << 12)):
        assert f(**kw) == B.ERR_INVALID_ARG, kw
    big = dict(rows=4096, k=4096, c_out=4096, stride=4096)
    need = L.cprune_mx4_linear_workspace_bytes(4096, 4096, 4096, 0)
    assert need > 0
    assert f(ws=None, **big) == f(size=need - 1, **big) == B.ERR_WORKSPACE
    assert f(ws=FAKE + 8, **big) == B.ERR_INVALID_ARG
    assert L.cprune_mx4_linear_workspace_bytes(0, 64, 8, 0) == 0


def test_the_convolutions_keep_their_activations():
    d = B.conv_desc((1, 8, 8, 8), (8, 8, 3, 3), 1, 1, act=B.ACT_SILU)
    assert B.lib().cprune_conv2d_bn_relu(d, FAKE, FAKE, None, None, FAKE, -1, None, 0, None) == B.ERR_INVALID_ARG


def test_the_binding_looks_at_its_tensors():
    x = torch.zeros(2, 3, 3, 8)
    with pytest.raises(ValueError):
        B.cprune_group_norm_act(x, 2)                     # not on the device
    with pytest.raises(ValueError):
        B.cprune_mx4_quantize(x)
    rows = B._rows_of
    assert rows(x, 1) == (2, 9, 8, 8)
    assert rows(x[..., :5], 1) == (2, 9, 5, 8)
    assert rows(x[:, :1, :1, :5], 1) == (2, 1, 5, 72)     # one pixel an image: images are the pixels' distance apart
    assert rows(x[:1, :1, :1, :3], 0) == (1, 1, 3, 3)
    assert rows(x.reshape(18, 8)[:, :3], 0) == (1, 18, 3, 8)
    with pytest.raises(ValueError):
        rows(x[:, :, ::2, :5], 1)                         # rows of the map end in a gap
    with pytest.raises(ValueError):
        rows(x.permute(0, 3, 1, 2), 1)                    # channels apart
    with pytest.raises(ValueError):
        rows(x[:, :1].expand(2, 3, 3, 8), 1)              # pixels on top of each other
    with pytest.raises(ValueError):
        rows(x.permute(0, 2, 1, 3)[..., :5], 1)           # pixels in another order


def test_norm_refuses_unaligned_scratch():
    L, d = B.lib(), _norm(n=2, pixels=1 << 16, c=12)
    odd = FAKE + 8
    assert L.cprune_group_norm_act(d, FAKE, None, None, FAKE, None, None, odd, 1 << 40, None) == B.ERR_INVALID_ARG
    assert L.cprune_group_norm_act_backward(d, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, None, odd, 1 << 40, None) == B.ERR_INVALID_ARG
