"""Where the calls on top logits, the distillation loss and the adapters get their memory when they are given a stream; needs no GPU."""
import pytest
import torch

from paper_2207_01260_amd import binding as B
from test_operator_streams import HERE, SIDE, on_device, world  # noqa: F401 (a fixture)


def calls():
    z, teacher, row = on_device(4, 30), on_device(4, 5), on_device(4)
    ids, labels = on_device(4, 5, dtype=torch.int32), on_device(4, dtype=torch.int32)
    stats = on_device(3, 4)
    x, a, b, base, scale = on_device(4, 12), on_device(2, 3, 12), on_device(2, 7, 3), on_device(4, 7), on_device(2)
    hidden, back = on_device(4, 3), on_device(4, 12)
    return {
        "top": (lambda **kw: B.cprune_top_logits(z, 5, **kw), [z]),
        "loss": (lambda **kw: B.cprune_distill_loss(z, ids, teacher, labels, hard=0.1, want_stats=True, **kw), [z, ids, teacher, labels]),
        "loss_grad": (lambda **kw: B.cprune_distill_loss_backward(row, z, ids, teacher, stats, labels, hard=0.1, **kw), [row, z, ids, teacher, stats, labels]),
        "step": (lambda **kw: B.cprune_distill_step(row, z, ids, teacher, labels, hard=0.1, **kw), [row, z, ids, teacher, labels]),
        "adapter": (lambda **kw: B.cprune_adapter_linear(x, a, b, labels, scale, base, want_hidden=True, **kw), [x, a, b, labels, scale, base]),
        "adapter_in_place": (lambda **kw: B.cprune_adapter_linear(x, a, b, labels, scale, base, out=base, **kw), [x, a, b, labels, scale, base]),
        "adapter_grad": (lambda **kw: B.cprune_adapter_linear_backward(base, x, hidden, a, b, labels, scale, back, **kw),
                         [base, x, hidden, a, b, labels, scale, back]),
    }


@pytest.mark.parametrize("name", sorted(calls()))
def test_memory_is_the_streams_and_is_kept_for_both(world, name):  # noqa: F811
    call, inputs = calls()[name]
    world.taken.clear()
    out = call(stream=SIDE)
    assert world.launched == [SIDE] and world.current == HERE
    assert world.taken and {s for s, _ in world.taken} == {SIDE}
    for t in out if isinstance(out, tuple) else (out,):
        assert (t.data_ptr(), HERE) in world.kept
    for t in inputs:
        assert (t.data_ptr(), SIDE) in world.kept


@pytest.mark.parametrize("name", sorted(calls()))
def test_without_a_stream_it_is_the_current_one(world, name):  # noqa: F811
    call, _ = calls()[name]
    world.taken.clear()
    call()
    assert world.launched == [HERE] and {s for s, _ in world.taken} == {HERE} and not world.kept


def test_what_is_not_wanted_takes_no_memory(world):  # noqa: F811
    x, a, b, dy, hidden = on_device(4, 12), on_device(2, 3, 12), on_device(2, 7, 3), on_device(4, 7), on_device(4, 3)
    world.taken.clear()
    dx, da, db = B.cprune_adapter_linear_backward(dy, x, hidden, a, b, want_weights=False, stream=SIDE)
    places = {at for _, at in world.taken}      # (a tensor may be listed twice)
    assert da is None and db is None and dx.data_ptr() in places and len(places) == 2
    world.taken.clear()
    dx, da, db = B.cprune_adapter_linear_backward(dy, x, hidden, a, b, want_dx=False, stream=SIDE)
    places = {at for _, at in world.taken}
    assert dx is None and {da.data_ptr(), db.data_ptr()} <= places and len(places) == 3
