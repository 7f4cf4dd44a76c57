"""The token model's step against the same model in 64 bits with automatic differentiation, and its training."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def reference_loss(P, model, ids, targets, old, adv, w, ref, kl):
    """The model's formulas on the FP16 weights, in 64 bits."""
    def norm(v):
        if model.kind:
            v = v - v.mean(1, keepdim=True)
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + model.eps)
    x = P["embed"][ids] * math.sqrt(model.D) * (ids != model.pad_id)[:, None]
    n = norm(x) * P["gain0"]
    for l in range(model.L):
        y = torch.relu(n @ P[f"w1.{l}"]) @ P[f"w2.{l}"]
        x = model.res * x + P[f"gate{l}"] * norm(y) * P[f"post{l}"]
        n = norm(x) * P[f"gain{l + 1}"]
    lp = torch.log_softmax(n @ P["out"], 1).gather(1, targets[:, None])[:, 0]
    r = torch.exp(lp - old.double())
    loss = -torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv)
    if ref is not None:
        d = ref.double() - lp
        loss = loss + kl * (torch.expm1(d) - d)
    return (w * loss).sum(), lp


@pytest.mark.parametrize("kind,V,D,F,n,kl", [(0, 101, 64, 128, 300, 0.0), (1, 29, 40, 72, 77, 0.1), (0, 9000, 128, 256, 64, 0.1)])
def test_gradients_match_automatic_differentiation(mp, kind, V, D, F, n, kl):
    from paper_1805_10387_b200.token_model import TokenModel
    model = TokenModel(V, D, F, 2, n, kind=kind, res_scale=0.9, pad_id=0, kl_coef=kl, init_scale=256.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    ids, targets = (torch.randint(0, V, (n,), generator=g, device="cuda") for _ in range(2))
    ids[7:12] = 0                                        # padding tokens, whose outputs do not count
    lp = torch.empty(n, device="cuda")
    model.log_probs(ids, targets, lp)
    old, ref, adv = lp + 0.02 * rnd(), (lp + 0.2 * rnd() if kl else None), rnd()
    w = torch.full((n,), 1.0 / n, device="cuda")
    w[ids == 0] = 0.0
    model.gradients(ids, targets, old, adv, w, ref)
    P = {k: v.double().requires_grad_() for k, v in model.w16.items()}
    loss, lp64 = reference_loss(P, model, ids, targets, old, adv.double(), w.double(), ref, kl)
    grads = dict(zip(P, torch.autograd.grad(loss, list(P.values()))))
    live = w != 0
    # FP16 activations of size about 1 between the calls: some 10 roundings of 2^-11 on the way to a log-probability
    assert (model.logp - lp64)[live].abs().max() < 0.05 and not model.logp[~live].any()
    assert abs(model.loss.item() - loss.item()) < 0.02
    for k, want in grads.items():
        got = model.dw[k].double() / 256.0
        off = (got - want).norm() / want.norm()
        assert off < 0.03, (k, off.item())
    h = model.state.read()
    assert h.found_inf == 0 and h.status == 0
    model.close()


def test_a_step_with_an_overflow_or_a_bad_token_changes_nothing(mp):
    from paper_1805_10387_b200.token_model import TokenModel
    n, V = 64, 50
    model = TokenModel(V, 64, 64, 1, n, init_scale=1024.0, state_bits=8)
    ids = torch.arange(n, device="cuda") % V
    z, one = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    lp = torch.empty(n, device="cuda")
    model.log_probs(ids, ids, lp)
    before = {k: v.clone() for k, v in model.w32.items()}
    same = lambda: all(torch.equal(before[k], v) for k, v in model.w32.items())  # noqa: E731
    model.step(ids, ids, lp, one * float("inf"), one)
    h = model.state.read()
    assert same() and h.skipped == 1 and h.t == 0 and h.scale == 512.0
    bad = ids.clone()
    bad[3] = V
    model.step(bad, ids, lp, one, one / n)
    assert same() and model.state.read().status == mp.MP_ERR_INVALID_ARG
    h.status = 0
    model.state.write(h)
    model.step(ids, ids, lp, one, one / n)
    assert not same() and model.state.read().t == 1
    # all tokens masked: no gradient, but the weights decay and the vectors stay
    before = {k: v.clone() for k, v in model.w32.items()}
    model.flat["m"][0].view(torch.uint8).zero_()
    model.step(ids, ids, lp, one, z)
    assert model.loss.item() == 0 and not model.dw["embed"].any()
    model.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_training_raises_the_rewarded_probability(mp, bits):
    from paper_1805_10387_b200.token_model import demo
    before, after = demo(steps=60, state_bits=bits)
    assert before < 0.1 and after > 0.5, (before, after)


def test_graph_replay_equals_eager_steps(mp):
    from paper_1805_10387_b200.token_model import TokenModel
    n, V = 200, 61
    g = torch.Generator(device="cuda").manual_seed(2)
    ids, targets = (torch.randint(0, V, (n,), generator=g, device="cuda") for _ in range(2))
    adv, w = torch.randn(n, generator=g, device="cuda"), torch.full((n,), 1.0 / n, device="cuda")
    models = [TokenModel(V, 64, 128, 2, n, init_scale=256.0, state_bits=8, seed=5) for _ in range(2)]
    old = torch.empty(n, device="cuda")
    models[0].log_probs(ids, targets, old)
    args = (ids, targets, old, adv, w)
    graph = models[0].capture(*args)
    for _ in range(3):
        graph.replay()
    for _ in range(4):
        models[1].step(*args)
    for k in models[0].w32:
        assert torch.equal(models[0].w32[k], models[1].w32[k]), k
    assert models[0].state.read().t == models[1].state.read().t == 4
    for m in models:
        m.close()
