"""What the top-logits and the distillation calls refuse, before anything is launched; needs no GPU."""
import math

import pytest
import torch

from paper_2207_01260_amd import binding as B

FAKE = 0x1000   # never dereferenced: validation fails first


def _top(z=FAKE, rows=4, classes=100, stride=100, k=5, dtype=0, values=FAKE, ids=FAKE, ws=FAKE, size=1 << 30):
    return B.lib().cprune_top_logits(z, rows, classes, stride, k, dtype, values, ids, ws, size, None)


@pytest.mark.parametrize("kw", [dict(z=None), dict(values=None), dict(ids=None), dict(rows=0), dict(rows=-1), dict(classes=0), dict(stride=99), dict(k=0), dict(k=-1),
                                dict(k=101), dict(dtype=3), dict(dtype=-1), dict(rows=1 << 16, classes=1 << 15, stride=1 << 15), dict(rows=3, stride=1 << 30),
                                dict(ws=FAKE + 8)])
def test_top_refuses(kw):
    assert _top(**kw) == B.ERR_INVALID_ARG


def test_top_refuses_more_than_it_does():
    L = B.lib()
    assert _top(k=257, classes=1000, stride=1000) == B.ERR_UNSUPPORTED
    assert _top(rows=1 << 22) == B.ERR_UNSUPPORTED
    assert L.cprune_top_logits_workspace_bytes(4, 1000, 257, 0) == L.cprune_top_logits_workspace_bytes(0, 1000, 5, 0) == 0
    need = L.cprune_top_logits_workspace_bytes(2, 1000000, 8, 1)
    assert need > 0
    long = dict(rows=2, classes=1000000, stride=1000000, k=8, dtype=1)
    assert _top(ws=None, **long) == _top(size=need - 1, **long) == B.ERR_WORKSPACE


def _desc(**kw):
    d = dict(rows=4, classes=100, k=5, dtype=B.F32, teacher_dtype=B.BF16, z_stride=100, temperature=2.0, hard=0.5)
    d.update(kw)
    return B.DistillDesc(*d.values())


def _calls(d, dloss=FAKE, z=FAKE, ids=FAKE, teacher=FAKE, loss=FAKE, stats=FAKE, dz=FAKE, ws=FAKE, size=1 << 30):
    L = B.lib()
    return {L.cprune_distill_loss(d, z, ids, teacher, None, loss, None, ws, size, None),
            L.cprune_distill_loss_backward(d, dloss, z, ids, teacher, None, stats, dz, None),
            L.cprune_distill_step(d, dloss, z, ids, teacher, None, loss, dz, ws, size, None)}


@pytest.mark.parametrize("kw", [dict(rows=0), dict(classes=0), dict(k=0), dict(dtype=3), dict(teacher_dtype=-1), dict(z_stride=99), dict(temperature=0.0),
                                dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=1e30), dict(temperature=1e-39),
                                dict(hard=-0.1), dict(hard=1.1), dict(hard=math.nan), dict(rows=1 << 16, classes=1 << 15, z_stride=1 << 15), dict(rows=3, z_stride=1 << 30)])
def test_distill_refuses(kw):
    d = _desc(**kw)
    assert _calls(d) == {B.ERR_INVALID_ARG}
    assert B.lib().cprune_distill_workspace_bytes(d) == 0


def test_distill_refuses_more_than_it_does_and_missing_pointers():
    assert _calls(_desc(k=257)) == _calls(_desc(rows=1 << 22)) == {B.ERR_UNSUPPORTED}
    assert _calls(None) == {B.ERR_INVALID_ARG}
    for name in ("z", "ids", "teacher"):
        assert _calls(_desc(), **{name: None}) == {B.ERR_INVALID_ARG}
    L, d = B.lib(), _desc()
    f = FAKE
    assert L.cprune_distill_loss(d, f, f, f, None, None, None, f, 1 << 30, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_loss_backward(d, None, f, f, f, None, f, f, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_loss_backward(d, f, f, f, f, None, None, f, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_loss_backward(d, f, f, f, f, None, f, None, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_step(d, None, f, f, f, None, f, f, f, 1 << 30, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_step(d, f, f, f, f, None, None, f, f, 1 << 30, None) == B.ERR_INVALID_ARG
    assert L.cprune_distill_step(d, f, f, f, f, None, f, None, f, 1 << 30, None) == B.ERR_INVALID_ARG
    long = _desc(rows=2, classes=100000, z_stride=100000)
    need = L.cprune_distill_workspace_bytes(long)
    assert need > 0
    assert L.cprune_distill_loss(long, f, f, f, None, f, None, None, 0, None) == L.cprune_distill_loss(long, f, f, f, None, f, None, f, need - 1, None) == B.ERR_WORKSPACE
    assert L.cprune_distill_step(long, f, f, f, f, None, f, f, f + 8, need, None) == B.ERR_INVALID_ARG


class OnDevice(torch.Tensor):
    is_cuda = True


def _on(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def test_binding_refuses_shapes_and_types():
    z, ids, t, y, w = _on(4, 10), _on(4, 3, dtype=torch.int32), _on(4, 3), _on(4, dtype=torch.int32), _on(4)
    stats = _on(3, 4)
    for bad in ((torch.zeros(4, 10), ids, t, y), (z, _on(4, 3, dtype=torch.int64), t, y), (z, _on(3, 3, dtype=torch.int32), t, y), (z, ids, _on(4, 2), y),
                (z, ids, _on(4, 3, dtype=torch.float64), y), (z, ids, t, _on(5, dtype=torch.int32)), (z, ids, t, _on(4, dtype=torch.int64)),
                (_on(4, 10, dtype=torch.int32), ids, t, y), (z, _on(3, 4, dtype=torch.int32).t(), t, y), (z, _on(dtype=torch.int32), t, y)):
        with pytest.raises(ValueError):
            B.cprune_distill_loss(*bad)
        with pytest.raises(ValueError):
            B.cprune_distill_step(w, *bad)
        with pytest.raises(ValueError):
            B.cprune_distill_loss_backward(w, *bad[:3], stats, bad[3])
    with pytest.raises(ValueError):
        B.cprune_distill_step(_on(5), z, ids, t, y)
    with pytest.raises(ValueError):
        B.cprune_distill_loss_backward(w, z, ids, t, _on(4, 3), y)
    for k in (0, 11, -1):
        with pytest.raises(ValueError):
            B.cprune_top_logits(z, k)
