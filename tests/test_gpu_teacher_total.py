"""The distillation loss over all rows against its formula in 64 bits.

Tolerance: a row's loss is off by 2^-20 of the magnitudes of its terms, and by three times what its log-probabilities are off by
(2^-20, and 2^-22 of the largest |z / temperature|); the sum over the rows, with at most 2^6 additions one after another, by 2^-18."""
import math

import pytest
import torch

from test_gpu_teacher import _distill, _gen, _rows, _teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("N,V,K,temp", [(1, 29, 4, 1.0), (700, 101, 8, 2.0), (3000, 1000, 20, 1.0), (300, 20000, 40, 0.7), (40, 131071, 128, 1.0)])
def test_total(mp, N, V, K, temp, tail):
    g = _gen(N + V)
    z = _rows(g, N, V)
    ids, a = _teacher(g, z, K, temp)
    w = torch.where(torch.rand(N, generator=g, device="cuda") < 0.7, torch.rand(N, generator=g, device="cuda") + 0.1, 0.0)
    w[0] = 1.0
    total = _distill(mp, z, ids, a, w, temp, tail)[2].double().item()
    x = z.double() / temp
    lq = torch.log_softmax(x, 1)
    la, a = lq.gather(1, ids), a.double()
    if not tail:
        a = torch.log_softmax(a, 1)
    p = a.exp()
    want, mag, mass = (p * (a - la)).sum(1), (p * (a.abs() + la.abs())).sum(1), p.sum(1)
    if tail:
        r, lr = 1 - mass, torch.logsumexp(lq.scatter(1, ids, -math.inf), 1)
        t = torch.where(r > 0, r * (r.clamp(min=1e-300).log() - lr), 0.0)
        # r is a difference of FP32 sums: off by 2^-22, and its logarithm with it
        want, mag, mass = want + t, mag + t.abs() + 1 + (r.clamp(min=2.0 ** -23).log() - lr).abs(), mass + r.clamp(min=0)
    rel = 2.0 ** -20 + x.abs().amax(1) * 2.0 ** -22
    want, tol = w.double() * want, w.double() * (mag * 2.0 ** -20 + mass * rel * 3)
    assert abs(total - want.sum().item()) <= tol.sum().item() + 2.0 ** -18 * want.abs().sum().item()
