"""The pointwise block on a stream of its caller's."""
import pytest
import torch

from paper_2207_01260_amd import pointwise, synth

pytestmark = pytest.mark.gpu


def test_a_block_on_a_stream_while_the_current_one_works():
    """Weights written by work that waits, a block built and run on another stream, tuned on the current one and run again, nothing waited for between."""
    values = torch.from_numpy(synth.tensor_normal((64, 40, 1, 1), 321, std=(2.0 / 40) ** 0.5)).cuda()
    x = torch.from_numpy(synth.tensor_normal((4, 14, 14, 40), 322)).cuda()

    def steps(stream, late):
        w, given = torch.zeros_like(values), torch.zeros_like(x)
        torch.cuda.synchronize()
        late()
        w.copy_(values)
        given.copy_(x)
        block = pointwise.PointwiseBlock(w, 45, 5, stream=stream)
        del w
        torch.zeros(64, 40, 1, 1, device="cuda")                # (what takes its place)
        late()
        first = block.forward(given, stream=stream)
        target = block.full(given) + 0.1
        late()
        errors = block.tune(given, target, 3, 1.0)
        second = block.forward(given, stream=stream)
        del given
        torch.zeros_like(x)
        late()
        out = [first + 0, second + 0, block.kept, block.codes, block.scales, block.weight, block.bias] + errors
        torch.cuda.synchronize()
        return out

    want = steps(None, lambda: None)
    side = torch.cuda.Stream()
    for _ in range(3):
        for late in (lambda: None, lambda: torch.cuda._sleep(10_000_000)):
            for got, expected in zip(steps(side, late), want):
                assert torch.equal(got, expected)
