"""Where the calls that take a stream get their memory, and for how long it is kept; needs no GPU: the library and torch's streams are stand-ins."""
import contextlib
import types

import pytest
import torch

from paper_2207_01260_amd import binding as B


HERE, SIDE = 16, 32


class OnDevice(torch.Tensor):
    is_cuda = True

    @property
    def device(self):
        return torch.device("cpu")


def on_device(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture()
def world(monkeypatch):
    """-> .current: the stream work goes to now; .taken: (stream, address) of every tensor made; .kept: (address, stream) that its memory waits for;
    .launched: the stream of every launch"""
    w = types.SimpleNamespace(current=HERE, taken=[], kept=set(), launched=[])

    @contextlib.contextmanager
    def stream(s):
        before, w.current = w.current, s
        yield
        w.current = before

    class Library:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return lambda *a: 256
            if name == "cprune_cached_tile":
                return lambda *a: B.ERR_INVALID_ARG
            return lambda *a: w.launched.append(getattr(a[-1], "value", a[-1])) or 0

    def made(f):
        def call(*a, **kw):
            t = f(*a, **kw).as_subclass(OnDevice)
            w.taken.append((w.current, t.data_ptr()))
            return t
        return call

    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_raw_stream", lambda s=None: w.current if s is None else s)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: w.current)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, made(getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "new_empty", made(torch.Tensor.new_empty))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.kept.add((t.data_ptr(), s)))
    return w


def calls():
    x, vec, stats = on_device(2, 5, 64), on_device(64), on_device(2, 4)
    w4, image, kept = on_device(5, 4, 3, 3), on_device(1, 4, 6, 6), on_device(3, dtype=torch.int32)
    codes, scales = on_device(10, 32, dtype=torch.uint8), on_device(10, 2, dtype=torch.uint8)
    return {
        "norm": (lambda **kw: B.cprune_group_norm_act(x, 4, vec, vec, want_stats=True, **kw), [x, vec]),
        "norm_grad": (lambda **kw: B.cprune_group_norm_act_backward(x, x, stats, stats, 4, vec, vec, **kw), [x, vec, stats]),
        "quantize": (lambda **kw: B.cprune_mx4_quantize(x, **kw), [x]),
        "dequantize": (lambda **kw: B.cprune_mx4_dequantize(codes, scales, 64, **kw), [codes, scales]),
        "matmul": (lambda **kw: B.cprune_mx4_matmul(codes, scales, codes, scales, B.F32, on_device(10), **kw), [codes, scales]),
        "linear": (lambda **kw: B.cprune_mx4_linear(x, codes, scales, on_device(10), **kw), [x, codes, scales]),
        "rank": (lambda **kw: B.cprune_rank_filters(w4, 3, **kw), [w4]),
        "rank_group": (lambda **kw: B.cprune_rank_filter_group([w4, w4], 3, **kw), [w4]),
        "gather": (lambda **kw: B.cprune_gather_pruned_weights(w4, kept, bn=(vec,) * 4, **kw), [w4, kept, vec]),
        "gather_channels": (lambda **kw: B.cprune_gather_channels(image, kept, **kw), [image, kept]),
        "conv": (lambda **kw: B.cprune_conv2d_bn_relu(B.conv_desc((1, 4, 6, 6), (5, 4, 3, 3)), image, w4, vec, **kw), [image, w4, vec]),
        "maxpool": (lambda **kw: B.cprune_maxpool2d(image, 2, 2, **kw), [image]),
        "avgpool": (lambda **kw: B.cprune_global_avgpool(image, **kw), [image]),
        "fc": (lambda **kw: B.cprune_fc(image, on_device(5, 144), **kw), [image]),
    }


@pytest.mark.parametrize("name", sorted(calls()))
def test_memory_is_the_streams_and_is_kept_for_both(world, name):
    call, inputs = calls()[name]
    world.taken.clear()
    out = call(stream=SIDE)
    assert world.launched == [SIDE] and world.current == HERE
    assert world.taken and {s for s, _ in world.taken} == {SIDE}
    for t in out if isinstance(out, tuple) else (out,):
        assert t is None or (t.data_ptr(), HERE) in world.kept
    for t in inputs:
        assert (t.data_ptr(), SIDE) in world.kept


@pytest.mark.parametrize("name", sorted(calls()))
def test_without_a_stream_it_is_the_current_one(world, name):
    call, _ = calls()[name]
    world.taken.clear()
    call()
    assert world.launched == [HERE] and {s for s, _ in world.taken} == {HERE} and not world.kept


@pytest.mark.parametrize("what", ["forward", "graph", "activation"])
def test_a_networks_outputs(world, monkeypatch, what):
    net = B.Net.__new__(B.Net)
    net._h, net._graph_logits, net.dtype, net.out_shape, net.out_features = None, {}, B.F32, (10,), 10
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    x = on_device(2, 3, 8, 8)
    world.taken.clear()
    out = net.activation(0, 2, (4, 8, 8), stream=SIDE) if what == "activation" else net.forward(x, use_graph=what == "graph", stream=SIDE)
    assert world.launched == [SIDE] and world.taken == [(SIDE, out.data_ptr())] and (out.data_ptr(), HERE) in world.kept
    if what != "activation":
        assert (x.data_ptr(), SIDE) in world.kept
    if what == "graph":
        assert net.forward(x, use_graph=True, stream=SIDE) is out
