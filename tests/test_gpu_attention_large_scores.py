"""Attention forward where scores are so large that FP32 holds them in steps of more than 1: the weights of a row still sum to 1.

With every value 1 an output is the sum of the rounded weights over the sum of the others: each weight is off by 2^-11 of itself, or by
2^-32 of the largest, the output rounds once (2^-11).  A log-sum is the largest score to FP32's rounding of score, factor and
exponent (three half steps of 2^-24 each), and the logarithm of at most n."""
import math

import pytest
import torch

from test_gpu_attention import Case, H

pytestmark = pytest.mark.gpu


def _large(power, D, n, step, sign):
    """Scores sign 2^power + step j for key j of n: 32 products of equal size, and one that changes from key to key."""
    c = Case([n], 1, 1, D, False, scale=1.0)
    a = 2.0 ** ((power - 5) // 2)
    c.q[:], c.k[:], c.v[:] = 0.0, 0.0, 1.0
    c.q[:, :32], c.k[:, :32] = a, sign * 2.0 ** (power - 5) / a
    c.q[:, 32] = step
    c.k[:, 32] = torch.arange(n, device="cuda").half()
    return c


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [10, 20, 21, 22, 23, 24, 25, 26, 27, 28, 30, 33])
def test_weights_sum_to_one(mp, power, D, sign):
    n = 300
    unit = 2.0 ** max(0, power - 23)                         # FP32's step there
    for step in sorted({0.0, 0.0625, 1.0, min(unit, 1024.0), min(2 * unit, 1024.0), min(4 * unit, 1024.0)}):
        c = _large(power, D, n, step, sign)
        c.forward(mp)
        assert bool(((c.o.double() - 1).abs() <= 2.1 * H + n * 2.0 ** -32).all()), (step, c.o.float().min().item(), c.o.float().max().item())
        x = (c.q.double() @ c.k.double().T).amax(1)
        # what FP32 keeps of the sum of products, in any order of its additions: 2 ^-23 of the magnitude for each of three roundings
        assert bool(((c.lse[0].double() - x).abs() <= 3 * 2.0 ** -23 * x.abs() + math.log(n) + 2.0 ** -18).all()), (step, (c.lse[0].double() - x).abs().max().item())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_large_queries_of_the_next_sequence_change_no_bits(mp, D, causal):
    for lengths in ([40, 300], [130, 70], [257, 5]):
        c = Case(lengths, 2, 1, D, causal, std=3.0, scale=8.0)
        c.forward(mp)
        n = lengths[0]
        o, lse = c.o[:n].clone(), c.lse[:, :n].clone()
        own = (c.q[:n].float().abs().max() * c.k[:n].float().abs().max() * D * 8).item()
        assert own < 2.0 ** 21                              # not large themselves
        for value in (60000.0, math.inf):
            c.q[n:] = value * c.k[0].sign().repeat(2)
            c.forward(mp)
            assert torch.equal(c.o[:n], o) and torch.equal(c.lse[:, :n], lse), (lengths, value)
