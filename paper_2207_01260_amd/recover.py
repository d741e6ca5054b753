"""A fully connected layer in 4 bits that a pruned network is brought back with: its codes stay, low-rank adapters beside them learn what the network answered
before, from the largest of its logits.

What Algorithm 1 does with a candidate before it is judged, some short training (line 10), on what a classifier in 4 bits has that may still change.  Several
variants, each with an adapter of its own, are served by one call on the same codes.
"""
from typing import List, Optional

import torch

from . import binding as B


class AdaptedLinear:
    """w [c_out, c], bias fp32 [c_out] or None, on the device: codes made once.  `variants` adapters of a rank, their first factor random from a seed, their second 0, so
    that the layer begins as its codes are.  They are kept in fp32 and multiplied in the type of x."""

    def __init__(self, w: torch.Tensor, bias: Optional[torch.Tensor] = None, rank: int = 8, variants: int = 1, scale: float = 1.0, seed: int = 0):
        c_out, c = w.shape
        self.codes, self.scales = B.cprune_mx4_quantize(w)
        self.bias = bias
        gen = torch.Generator().manual_seed(seed)
        self.a = (torch.randn(variants, rank, c, generator=gen) * c ** -0.5).to(w.device)
        self.b = torch.zeros(variants, c_out, rank, device=w.device)
        self.scale = torch.full((variants,), scale, device=w.device)

    def forward(self, x: torch.Tensor, which: Optional[torch.Tensor] = None, want_hidden: bool = False):
        """x [..., c] -> logits [..., c_out]; which int32 [...]: each row's variant (-1: the codes alone).  (logits, hidden) for `gradients`."""
        base = B.cprune_mx4_linear(x, self.codes, self.scales, self.bias)
        return B.cprune_adapter_linear(x, self.a.to(x.dtype), self.b.to(x.dtype), which, self.scale, base, want_hidden=want_hidden, out=base)

    def gradients(self, x: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, labels: Optional[torch.Tensor] = None,
                  which: Optional[torch.Tensor] = None, temperature: float = 2.0, hard: float = 0.0):
        """-> (the rows' losses, fp32; gradients of their mean by the adapters' factors, fp32)."""
        z, hidden = self.forward(x, which, want_hidden=True)
        # A row's share of the mean would be below fp16's normal numbers from some thousand rows on: the power of two that brings it to between a half and one is taken out
        # again of the factors' gradients.  (The other types' bits are the same either way.)
        rows = z.numel() // z.shape[-1]
        up = 2.0 ** (rows.bit_length() - 1)
        share = torch.full(z.shape[:-1], up / rows, device=z.device)
        loss, dz = B.cprune_distill_step(share, z, ids, teacher, labels, temperature, hard)
        _, da, db = B.cprune_adapter_linear_backward(dz, x, hidden, self.a.to(x.dtype), self.b.to(x.dtype), which, self.scale, want_dx=False)
        return loss, da / up, db / up

    def tune(self, x: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, steps: int, rate: float, **kw) -> List[torch.Tensor]:
        """Gradient descent on the adapters; -> the mean loss of every step."""
        losses = []
        for _ in range(steps):
            loss, da, db = self.gradients(x, ids, teacher, **kw)
            self.a -= rate * da
            self.b -= rate * db
            losses.append(loss.mean())
        return losses
