"""Attention forward where a row's largest weight hides thousands of small ones.

Tolerances, from the roundings: a weight enters its product in FP16, times 2^7 and in units of the row's largest (or of a running
maximum below it): half a step of 2^-11 of it, or 2^-25 where the product with 2^7 is subnormal, which is 2^-32 of the largest.  An
output is rounded once (2^-11 of it, 2^-25 where it is subnormal).  A score is an FP32 sum of D products (D 2^-23 of the sum of their
magnitudes with its exponent's rounding).  Sums over n keys: n / 16 additions of the tensor core and n / 64 of a row's sum, each at
most 2^-23 of the sum of magnitudes."""
import math

import pytest
import torch

from test_gpu_attention import Case, H

pytestmark = pytest.mark.gpu


def check_rows(c, rows, h=0):
    """The outputs of some rows (indices within the only sequence) of head h."""
    n, D = c.lengths[0], c.D
    b = slice(h * c.hk // c.hq * D, (h * c.hk // c.hq + 1) * D)
    a = slice(h * D, (h + 1) * D)
    for i in rows.split(max(1, 2 ** 25 // n)):
        q, k, v = c.q[c.before + i, a].double(), c.k[c.before:c.before + n, b].double(), c.v[c.before:c.before + n, b].double()
        gap = i[:, None] - torch.arange(n, device="cuda")
        seen = torch.ones_like(gap, dtype=torch.bool)
        if c.causal:
            seen = gap >= 0
            if c.window:
                seen &= gap < c.window
        x = (q @ k.T * c.scale).masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(x, 1)
        p = (x - lse[:, None]).exp()
        es = (q.abs() @ k.abs().T).masked_fill(~seen, 0).amax(1, keepdim=True) * c.scale * D * 2.0 ** -23 + 2.0 ** -20
        most = p.amax(1, keepdim=True)
        e_p = torch.where(p >= 2.0 ** -21 * most, H * p, 2.0 ** -32 * most) * seen
        o, mag = p @ v, p @ v.abs()
        sums = (n / 16 + 32) * 2.0 ** -23
        tol = 1.01 * (e_p @ v.abs() + H * o.abs()) + (2 * es + sums) * mag + 2.0 ** -25
        err = (c.o[c.before + i, a].double() - o).abs()
        assert bool((err <= tol).all()), (h, (err / tol).max().item())
        err = (c.lse[h, c.before + i].double() - lse).abs()
        assert bool((err <= es[:, 0] + sums + 2.0 ** -22 * lse.abs()).all()), (h, err.max().item())


@pytest.mark.parametrize("n,D,causal", [(1000, 64, False), (16385, 64, True), (16385, 128, True), (16385, 72, False), (131073, 64, True)])
@pytest.mark.parametrize("nats", [8.0, 12.0, 18.0])
def test_one_key_above_many(mp, nats, n, D, causal):
    """The first key, whose value is 0, holds nearly all of a row; what comes out is what the others weigh."""
    c = Case([n], 1, 1, D, causal, scale=1.0)
    c.q *= 0.3
    c.k *= 0.1
    c.q[:, 0], c.k[:, 0], c.v[:] = 6.0, 0.0, 1 + 0.5 * c.v
    c.k[0, 0], c.v[0] = nats / 6.0, 0.0
    c.forward(mp)
    check_rows(c, torch.cat([torch.arange(0, n, max(1, n // 100), device="cuda"), torch.arange(n - 130, n, device="cuda")]))
