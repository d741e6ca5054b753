"""Where the calls that take a stream get their memory, and for how long it is kept; needs no GPU: the library and torch's streams are stand-ins."""
import contextlib
import types

import pytest
import torch

from paper_2207_01260_amd import binding as B


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
    w = types.SimpleNamespace(current="here", taken=[], kept=set(), launched=[])

    @contextlib.contextmanager
    def stream(s):
        before, w.current = w.current, s
        yield
        w.current = before

    class Library:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return lambda *a: 256
            return lambda *a: w.launched.append(a[-1]) or 0

    def made(f):
        def call(*a, **kw):
            t = f(*a, **kw)
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
    codes, scales = on_device(10, 32, dtype=torch.uint8), on_device(10, 2, dtype=torch.uint8)
    return {
        "norm": (lambda **kw: B.cprune_group_norm_act(x, 4, vec, vec, want_stats=True, **kw), [x, vec]),
        "norm_grad": (lambda **kw: B.cprune_group_norm_act_backward(x, x, stats, stats, 4, vec, vec, **kw), [x, vec, stats]),
        "quantize": (lambda **kw: B.cprune_mx4_quantize(x, **kw), [x]),
        "dequantize": (lambda **kw: B.cprune_mx4_dequantize(codes, scales, 64, **kw), [codes, scales]),
        "matmul": (lambda **kw: B.cprune_mx4_matmul(codes, scales, codes, scales, B.F32, on_device(10), **kw), [codes, scales]),
        "linear": (lambda **kw: B.cprune_mx4_linear(x, codes, scales, on_device(10), **kw), [x, codes, scales]),
    }


@pytest.mark.parametrize("name", sorted(calls()))
def test_memory_is_the_streams_and_is_kept_for_both(world, name):
    call, inputs = calls()[name]
    world.taken.clear()
    out = call(stream="side")
    assert world.launched == ["side"] and world.current == "here"
    assert world.taken and {s for s, _ in world.taken} == {"side"}
    for t in out if isinstance(out, tuple) else (out,):
        assert (t.data_ptr(), "here") in world.kept
    for t in inputs:
        assert (t.data_ptr(), "side") in world.kept


@pytest.mark.parametrize("name", sorted(calls()))
def test_without_a_stream_it_is_the_current_one(world, name):
    call, _ = calls()[name]
    world.taken.clear()
    call()
    assert world.launched == ["here"] and {s for s, _ in world.taken} == {"here"} and not world.kept
