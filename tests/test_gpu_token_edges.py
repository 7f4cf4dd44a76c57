"""Values at the edges of what FP32 holds, and orders of calls, that the token-model operators have to get right."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("V", [29, 700, 20000])
def test_a_ratio_past_fp32_times_a_zero_factor_is_zero(mp, V):
    """exp(lp - old_logp) and exp(ref_logp - lp) of 2.7e43 pass FP32, but they are finite, and 0 times them is 0: an
    advantage of 0 gives no loss, and a KL factor of 0 no KL term."""
    N = 6
    z, dz = (torch.zeros(N, -(-V // 8) * 8, dtype=torch.float16, device="cuda")[:, :V] for _ in range(2))
    t = torch.arange(N, device="cuda")
    lp = torch.full((N,), -math.log(V), device="cuda")
    adv = torch.tensor([0.0, -0.0, 0.0, 1.0, -1.0, 0.0], device="cuda")
    old = lp - 100.0
    old[2] = lp[2]
    old[5] = float("nan")
    ref = lp + 100.0
    w = torch.ones(N, device="cuda")
    for clip_hi in (0.25, float("inf")):
        for with_ref in (False, True):
            dz.fill_(7.0)
            got, tl = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
            mp.mp_policy_loss(z, t, old, adv, w, got, tl, dlogits16=dz, ref_logp=ref if with_ref else None, clip_lo=0.25,
                              clip_hi=clip_hi, kl_coef=0.0)
            assert not tl[:3].any() and not dz[:3].any(), (clip_hi, with_ref)
            # 1.25 A where the ratio is clipped from above (then without a gradient); what passes FP32 is an infinity
            assert tl[3].item() == (-1.25 if clip_hi == 0.25 else -math.inf) and tl[4].item() == math.inf
            assert clip_hi != 0.25 or not dz[3].any()
            assert torch.isnan(tl[5]) and torch.isnan(dz[5]).all()                  # a NaN shows whatever the advantage is
    mp.mp_policy_loss(z, t, lp, adv, w, got, tl, dlogits16=dz, ref_logp=ref, kl_coef=0.1)    # a KL term that is meant
    assert (tl == math.inf).all()
