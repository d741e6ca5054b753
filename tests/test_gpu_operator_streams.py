"""The calls on a stream beside one that is still at work: they write nothing that its work reads."""
import pytest
import torch

from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu


def test_memory_that_the_current_stream_still_reads():
    """A tensor is read by work that waits, and given back: what a call on another stream writes meanwhile is other memory."""
    rows, k, c_out, groups = 512, 768, 768, 8
    x = torch.randn(rows, k, device="cuda")
    wc, ws = B.cprune_mx4_quantize(torch.randn(c_out, k, device="cuda"))
    codes = B.cprune_mx4_quantize(x)
    weight, bias = torch.rand(k, device="cuda"), torch.rand(k, device="cuda")
    maps = x.reshape(4, 128, k)
    _, mean, rstd = B.cprune_group_norm_act(maps, groups, weight, bias, want_stats=True)
    side = torch.cuda.Stream()
    for call in (lambda **kw: B.cprune_mx4_linear(x, wc, ws, **kw), lambda **kw: B.cprune_mx4_matmul(*codes, wc, ws, B.F32, **kw),
                 lambda **kw: B.cprune_mx4_dequantize(*codes, k, **kw), lambda **kw: B.cprune_mx4_quantize(x, **kw)[0],
                 lambda **kw: B.cprune_group_norm_act(maps, groups, weight, bias, **kw),
                 lambda **kw: B.cprune_group_norm_act_backward(maps, maps, mean, rstd, groups, weight, bias, **kw)[0]):
        want = call()
        kept = torch.empty_like(want)
        torch.cuda.synchronize()
        for _ in range(3):
            old = torch.full_like(want, 7)          # the size of the call's output
            torch.cuda._sleep(20_000_000)           # some ten milliseconds
            kept.copy_(old)
            del old
            got = call(stream=side)
            side.synchronize()
            torch.cuda.synchronize()
            assert bool((kept == 7).all()) and torch.equal(got, want)
            del got
