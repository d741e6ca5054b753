"""A pointwise block of a channel-pruned network in 4 bits: group norm, SiLU and a 1x1 convolution on microscaled codes.

Pruning takes filters out (Section 3.5 of the paper, last paragraph); what is left of a 1x1 layer is stored and multiplied as 4-bit codes.  Such a
block has few numbers that may still change: weight and bias of its norm.  They are tuned as the paper tunes a pruned candidate, for a few
steps on a few images (Section 3.2), against what the block answered before its weights became codes: forward through the codes, backward
through the numbers that the weights' codes stand for (the rounding of the activations passes gradients on unchanged) and through the norm.

    python -m paper_2207_01260_amd.pointwise [--c-in 96] [--c-out 128] [--keep 83] [--hw 14] [--batch 8] [--steps 40]

prints the mean squared error before and after, relative to the answers' own, and the time of a forward pass.
"""
import argparse
import math

import torch

from . import binding as B
from . import synth


def _between(stream, call, *args):
    """call(*args) on `stream`, between what torch's current stream has had and what it gets."""
    here = torch.cuda.current_stream()
    stream.wait_stream(here)
    with torch.cuda.stream(stream):
        out = call(*args)
    here.wait_stream(stream)
    return out


class PointwiseBlock:
    """x [n, h, w, c] channels last -> [n, h, w, filters kept].  w: the 1x1 layer's raw weights, fp32 [c_out][c][1][1] on the device; its `keep` strongest
    filters survive.

    What is given a `stream` runs there, behind what the current stream has been given so far and ahead of what it is given next: the block's weights are one
    set, which `tune` changes on the current stream.  The other calls run on the current stream."""

    def __init__(self, w: torch.Tensor, keep: int, groups: int, act: int = B.ACT_SILU, stream=None):
        self.groups, self.act = groups, act
        if stream is None:
            self._build(w, keep)
        else:
            for t in _between(stream, self._build, w, keep):
                t.record_stream(torch.cuda.current_stream())

    def _build(self, w: torch.Tensor, keep: int):
        c = w.shape[1]
        _, _, self.kept = B.cprune_rank_filters(w, keep, want_scores=False, want_order=False)
        kept_w, _ = B.cprune_gather_pruned_weights(w, self.kept)
        self.w = kept_w.reshape(keep, c)
        self.codes, self.scales = B.cprune_mx4_quantize(self.w)
        self.weight = torch.ones(c, device=w.device)
        self.bias = torch.zeros(c, device=w.device)
        return self.kept, self.w, self.codes, self.scales, self.weight, self.bias

    def forward(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        if stream is not None:
            y = _between(stream, self.forward, x)
            y.record_stream(torch.cuda.current_stream())
            return y
        z = B.cprune_group_norm_act(x, self.groups, self.weight, self.bias, act=self.act)
        return B.cprune_mx4_linear(z, self.codes, self.scales)

    def full(self, x: torch.Tensor) -> torch.Tensor:
        """The block's answer with its weights as they were."""
        z = B.cprune_group_norm_act(x, self.groups, self.weight, self.bias, act=self.act)
        y = B.cprune_fc(z.reshape(-1, z.shape[-1]), self.w.to(z.dtype))
        return y.reshape(z.shape[:-1] + (y.shape[-1],))

    def gradients(self, x: torch.Tensor, target: torch.Tensor):
        """-> (mean squared error against target, its gradients by the norm's weight and bias and by x, in fp32)."""
        z, mean, rstd = B.cprune_group_norm_act(x, self.groups, self.weight, self.bias, act=self.act, want_stats=True)
        y = B.cprune_mx4_linear(z, self.codes, self.scales)
        miss = y.float() - target.float()
        # An answer's share, 2 / count, is below fp16's normal numbers from 33000 answers on: the power of two that brings it to between a half and one is taken
        # out again behind the norm.  (The other types' bits are the same either way.)
        up = 2.0 ** math.floor(math.log2(miss.numel() / 2.0))
        dy = (miss * (2.0 / miss.numel() * up)).to(x.dtype)
        c = x.shape[-1]
        # dz = dy w: a fully connected layer with the decoded weights' transpose as its weights
        back = B.cprune_mx4_dequantize(self.codes, self.scales, c, B.DTYPE_OF_TORCH[x.dtype]).t().contiguous()
        dz = B.cprune_fc(dy.reshape(-1, dy.shape[-1]), back).reshape(x.shape)
        dx, dweight, dbias = B.cprune_group_norm_act_backward(dz, x, mean, rstd, self.groups, self.weight, self.bias, act=self.act)
        return miss.square().mean(), dweight / up, dbias / up, dx.float() / up

    def tune(self, x: torch.Tensor, target: torch.Tensor, steps: int, rate: float):
        """Gradient descent on the norm's vectors; -> the error of every step."""
        errors = []
        for _ in range(steps):
            error, dweight, dbias, _ = self.gradients(x, target)
            self.weight -= rate * dweight
            self.bias -= rate * dbias
            errors.append(error)
        return errors


def run(c_in=96, c_out=128, keep=83, hw=14, batch=8, steps=40, groups=8, rate=1.0, dtype=B.F32):
    """-> (errors of the steps relative to the answers' mean square, microseconds of a forward pass)."""
    w = torch.from_numpy(synth.tensor_normal((c_out, c_in, 1, 1), 301, c_out, c_in, std=(2.0 / c_in) ** 0.5)).cuda()
    x = torch.from_numpy(synth.tensor_normal((batch, hw, hw, c_in), 302, batch, hw)).cuda().to(B.TORCH_DTYPE[dtype])
    block = PointwiseBlock(w, keep, groups)
    target = block.full(x)
    scale = float(target.float().square().mean())
    errors = [float(e) / scale for e in block.tune(x, target, steps, rate)]
    block.forward(x)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(50):
        block.forward(x)
    end.record()
    torch.cuda.synchronize()
    return errors, start.elapsed_time(end) / 50 * 1e3


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("--c-in", 96), ("--c-out", 128), ("--keep", 83), ("--hw", 14), ("--batch", 8), ("--steps", 40), ("--groups", 8)):
        ap.add_argument(name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=1.0)
    args = ap.parse_args()
    errors, us = run(args.c_in, args.c_out, args.keep, args.hw, args.batch, args.steps, args.groups, args.rate)
    print(f"error of the 4-bit block {errors[0]:.5f} of the answers' mean square, after {len(errors)} steps {errors[-1]:.5f}; forward {us:.1f} us")


if __name__ == "__main__":
    main()
