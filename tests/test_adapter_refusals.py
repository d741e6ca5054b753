"""What the adapter calls refuse, before anything is launched; needs no GPU."""
import pytest
import torch

from paper_2207_01260_amd import binding as B

FAKE = 0x1000   # never dereferenced: validation fails first


def _desc(**kw):
    d = dict(rows=70, k=40, c_out=30, rank=8, adapters=3, dtype=B.F16, act=0, mixed=1, x_stride=40, base_stride=40, dy_stride=30)
    d.update(kw)
    return B.AdapterDesc(*d.values())


def _forward(d, x=FAKE, a=FAKE, b=FAKE, which=FAKE, scale=None, base=None, y=FAKE, hidden=None, ws=FAKE, size=1 << 40):
    return B.lib().cprune_adapter_linear(d, x, a, b, which, scale, base, y, hidden, ws, size, None)


def _backward(d, dy=FAKE, x=FAKE, hidden=FAKE, a=FAKE, b=FAKE, which=FAKE, scale=None, base=None, dx=FAKE, da=FAKE, db=FAKE, ws=FAKE, size=1 << 40):
    return B.lib().cprune_adapter_linear_backward(d, dy, x, hidden, a, b, which, scale, base, dx, da, db, ws, size, None)


BAD = [dict(rows=0), dict(k=0), dict(c_out=0), dict(rank=0), dict(adapters=0), dict(rows=-1), dict(dtype=3), dict(dtype=-1), dict(mixed=2), dict(mixed=-1),
       dict(x_stride=39), dict(rows=1 << 20, x_stride=1 << 11), dict(rows=1 << 20, c_out=1 << 11, dy_stride=1 << 11), dict(rows=1 << 29),
       dict(adapters=1000, rank=100, k=1 << 15, x_stride=1 << 15), dict(adapters=1000, rank=100, c_out=1 << 15, dy_stride=1 << 15)]


@pytest.mark.parametrize("kw", BAD + [dict(act=4), dict(act=-1)])
def test_forward_refuses(kw):
    d = _desc(**kw)
    assert _forward(d) == B.ERR_INVALID_ARG
    assert B.lib().cprune_adapter_workspace_bytes(d, 0) == 0


@pytest.mark.parametrize("kw", BAD + [dict(dy_stride=29)])
def test_backward_refuses(kw):
    d = _desc(**kw)
    assert _backward(d) == B.ERR_INVALID_ARG
    assert B.lib().cprune_adapter_workspace_bytes(d, 1) == 0


def test_more_than_they_do():
    for kw in (dict(rank=129), dict(adapters=1025)):
        assert _forward(_desc(**kw)) == _backward(_desc(**kw)) == B.ERR_UNSUPPORTED
        assert B.lib().cprune_adapter_workspace_bytes(_desc(**kw), 0) == B.lib().cprune_adapter_workspace_bytes(_desc(**kw), 1) == 0
    wide = _desc(rows=(1 << 31) - 1, k=1, c_out=1, rank=1, x_stride=1, dy_stride=1, adapters=1, mixed=0)      # (more places than 32 bits count)
    assert _forward(wide) == _backward(wide) == B.ERR_UNSUPPORTED


def test_missing_pointers_and_scratch():
    d = _desc()
    for name in ("x", "a", "b", "which", "y"):
        assert _forward(d, **{name: None}) == B.ERR_INVALID_ARG
    for name in ("dy", "a", "b", "which", "x", "hidden", "da", "db"):
        assert _backward(d, **{name: None}) == B.ERR_INVALID_ARG
    assert _backward(d, dx=None, da=None, db=None) == B.ERR_INVALID_ARG
    assert _forward(None) == _backward(None) == B.ERR_INVALID_ARG
    assert _forward(_desc(base_stride=29), base=FAKE) == B.ERR_INVALID_ARG
    assert _forward(_desc(base_stride=31), base=FAKE, y=FAKE) == B.ERR_INVALID_ARG       # (in place, but not dense)
    assert _backward(_desc(base_stride=39), base=FAKE) == B.ERR_INVALID_ARG
    assert _backward(_desc(base_stride=41), base=FAKE, dx=FAKE) == B.ERR_INVALID_ARG
    for call, back in ((_forward, 0), (_backward, 1)):
        need = B.lib().cprune_adapter_workspace_bytes(d, back)
        assert need > 0
        assert call(d, ws=None) == call(d, size=need - 1) == B.ERR_WORKSPACE
        assert call(d, ws=FAKE + 8) == B.ERR_INVALID_ARG


class OnDevice(torch.Tensor):
    is_cuda = True


def _on(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def test_binding_refuses_shapes_and_types():
    x, a, b, which, scale, base = _on(5, 12), _on(2, 4, 12), _on(2, 7, 4), _on(5, dtype=torch.int32), _on(2), _on(5, 7)
    dy, hidden, dx = _on(5, 7), _on(5, 4), _on(5, 12)
    for bad in ((torch.zeros(5, 12), a, b, which, scale, base), (x, _on(4, 12), b, which, scale, base), (x, a, _on(7, 4), which, scale, base),
                (x, _on(2, 4, 11), b, which, scale, base), (x, a, _on(3, 7, 4), which, scale, base), (x, a, _on(2, 7, 5), which, scale, base),
                (x, _on(2, 4, 12, dtype=torch.float16), b, which, scale, base), (x, a, b, _on(5, dtype=torch.int64), scale, base), (x, a, b, _on(4, dtype=torch.int32), scale, base),
                (x, a, b, which, _on(3), base), (x, a, b, which, scale, _on(5, 8)), (x, a, b, which, scale, _on(5, 7, dtype=torch.bfloat16)),
                (x, a, b, which, scale, torch.zeros(5, 7)), (_on(5, 12, dtype=torch.float64), a, b, which, scale, base), (x, a.transpose(1, 2), b, which, scale, base)):
        with pytest.raises(ValueError):
            B.cprune_adapter_linear(*bad)
    for out in (_on(5, 8), _on(5, 7, dtype=torch.float16), _on(7, 5).t(), torch.zeros(5, 7)):
        with pytest.raises(ValueError):
            B.cprune_adapter_linear(x, a, b, out=out)
    for bad in ((_on(5, 8), x, hidden), (dy, x, _on(5, 5)), (dy, x, _on(5, 4, dtype=torch.float16)), (_on(4, 7), x, hidden), (torch.zeros(5, 7), x, hidden)):
        with pytest.raises(ValueError):
            B.cprune_adapter_linear_backward(*bad, a, b, which, scale, dx)
    with pytest.raises(ValueError):
        B.cprune_adapter_linear_backward(dy, x, hidden, a, b, which, scale, _on(5, 13))
