"""The distillation loss over rows so long that a thread adds thousands of numbers, hardly any two of them different: a single chain of n equal ones in 32 bits is off by up to n / 4
units of e = 2^-24.

A row holds 0 in the first 4096 of every 65536 places, so that every thread meets it, and -d in the others: its sums have a closed form.  Bounds: chains of at most 264 numbers (256 and a row's edge), 64 such chains at most, joined in
another, and 16 steps over lanes, wavefronts and parts: 344 e of a sum, its terms (3 d + 2) e each, a logarithm 2 e of itself more.  A probability is off by that of its sum and
of its term, a stored logarithm by e of itself for each unit of it; gradients are rounded to the type, u."""
import math

import pytest
import torch

from paper_2207_01260_amd import binding as B

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


# rows of a work-group each, and few rows that are cut; 4096 to 8192 numbers a thread
@pytest.mark.parametrize("rows,classes,dtype", [(128, (1 << 21) + 5, torch.bfloat16), (128, 1 << 20, torch.float32), (3, (1 << 26) + 9, torch.float16)])
@pytest.mark.parametrize("temperature", [1.0, 2.0, 3.0])
def test_long_chains(rows, classes, dtype, temperature):
    T, hard = temperature, 0.5
    d = 0.25 + torch.arange(rows, device="cuda", dtype=torch.float32) / 32 if rows > 3 else torch.tensor([0.59375, 3.40625, 1.9375], device="cuda")
    z = (-d).to(dtype)[:, None].repeat(1, classes)      # (numbers of the type)
    zeros = torch.arange(classes, device="cuda") % 65536 < 4096
    z[:, zeros] = 0
    zero = int(zeros.sum())
    ids = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    teacher = torch.ones(rows, 1, dtype=dtype, device="cuda")
    labels = torch.full((rows,), 5000, dtype=torch.int32, device="cuda")
    dloss = torch.full((rows,), 1.0, device="cuda")
    loss, stats = B.cprune_distill_loss(z, ids, teacher, labels, T, hard, want_stats=True)
    step, dz = B.cprune_distill_step(dloss, z, ids, teacher, labels, T, hard)
    places = torch.tensor([0, 5000, 5001, classes - 1], device="cuda")
    dz = dz[:, places].double().cpu()
    back = B.cprune_distill_loss_backward(dloss, z, ids, teacher, stats, labels, T, hard)[:, places].double().cpu()
    loss, stats, step = loss.double().cpu(), stats.double().cpu(), step.double().cpu()
    for r in range(rows):
        far = float(d[r])
        s = [zero + (classes - zero) * math.exp(-far / t) for t in (T, 1.0)]
        log = [math.log(v) for v in s]
        off = [(344 + 3 * far / t + 2 + 2 * v) * E for t, v in zip((T, 1.0), log)]
        for i in range(2):
            assert abs(stats[1 + i, r] - log[i]) <= off[i], (r, i)
        # p is 1: (1 - h) T^2 (0 - log q_T of the largest) and h (log of the sum + d)
        want = (1 - hard) * T * T * log[0] + hard * (log[1] + far)
        bound = (1 - hard) * T * T * off[0] + hard * off[1] + 8 * E * want
        assert abs(loss[r] - want) <= bound and abs(step[r] - want) <= bound, r
        for j, place in enumerate((0, 5000, 5001, classes - 1)):
            e = far if place % 65536 >= 4096 else 0.0
            q, one = math.exp(-e / T) / s[0], math.exp(-e) / s[1]
            want = (1 - hard) * T * (q - (place == 0)) + hard * (one - (place == 5000))
            bound = (1 - hard) * T * q * (off[0] + 8 * E) + hard * one * (off[1] + 8 * E) + 4 * E * ((1 - hard) * T * (place == 0) + hard * (place == 5000))
            bound = bound * (1 + U[dtype]) + U[dtype] * abs(want) + (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -120)
            assert abs(dz[r, j] - want) <= bound and abs(back[r, j] - want) <= bound, (r, place)
