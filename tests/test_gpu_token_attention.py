"""The token model with attention and with distillation: whole gradients against the same model in 64 bits with automatic
differentiation, replayed steps, and the demonstration."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def logits64(P, model, ids, lengths):
    """The model's formulas on the FP16 weights, in 64 bits."""
    def norm(v, layer=model.kind):
        if layer:
            v = v - v.mean(-1, keepdim=True)
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + model.eps)

    def turn(v):
        rot = 0 if model.freqs is None else 2 * len(model.freqs)
        t = model.positions.double()[:, None, None] * (model.freqs if rot else 0)
        a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        return torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos(), v[..., rot:]], 2) if rot else v
    hq, hk, hd = model.hq, model.hk, model.hd
    x = P["embed"][ids] * math.sqrt(model.D) * (ids != model.pad_id)[:, None]
    n = norm(x) * P["gain0"]
    for l in range(model.L):
        qkv = (n @ P[f"qkv.{l}"]).view(model.n, -1, hd)
        q, k = turn(norm(qkv[:, :hq], 0) * P[f"gq{l}"]), turn(norm(qkv[:, hq:hq + hk], 0) * P[f"gk{l}"])
        v, outs, at = qkv[:, hq + hk:], [], 0
        for m in lengths:
            r = slice(at, at + m)
            at += m
            gap = torch.arange(m, device="cuda")[:, None] - torch.arange(m, device="cuda")
            hidden = (gap < 0) | (gap >= model.window) if model.window else gap < 0
            one = [torch.softmax((q[r, h] @ k[r, h * hk // hq].T / math.sqrt(hd)).masked_fill(hidden, -math.inf), 1)
                   @ v[r, h * hk // hq] for h in range(hq)]
            outs.append(torch.stack(one, 1))
        y = torch.cat(outs).reshape(model.n, -1) @ P[f"attn_out.{l}"]
        x = model.res * x + P[f"agate{l}"] * norm(y) * P[f"apost{l}"]
        n = norm(x) * P[f"again{l}"]
        y = torch.relu(n @ P[f"w1.{l}"]) @ P[f"w2.{l}"]
        x = model.res * x + P[f"gate{l}"] * norm(y) * P[f"post{l}"]
        n = norm(x) * P[f"gain{l + 1}"]
    return n @ P["out"]


def distill64(z, ids, a, w, temp, tail):
    lq = torch.log_softmax(z / temp, 1)
    a, la = a.double(), lq.gather(1, ids.long())
    if not tail:
        a = torch.log_softmax(a, 1)
        return (w * (a.exp() * (a - la)).sum(1)).sum()
    rest = torch.logsumexp(lq.scatter(1, ids.long(), -math.inf), 1)
    r = 1 - a.exp().sum(1)
    return (w * ((a.exp() * (a - la)).sum(1) + r * (r.log() - rest))).sum()


@pytest.mark.parametrize("kind,V,hq,hk,hd,window,tail,lengths", [
    (0, 101, 4, 2, 32, 0, True, [150, 1, 149]), (1, 300, 2, 2, 64, 20, False, [200]), (0, 3000, 3, 1, 40, 0, True, [130, 0, 37])])
def test_gradients_match_automatic_differentiation(mp, kind, V, hq, hk, hd, window, tail, lengths):
    from paper_1805_10387_b200.token_model import TokenModel
    n, D, k, temp = sum(lengths), 64, 10, 1.5
    model = TokenModel(V, D, 128, 2, n, kind=kind, res_scale=0.9, init_scale=512.0, heads=hq, kv_heads=hk, head_dim=hd, window=window,
                       sequences=4)
    model.set_sequences(lengths)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    teacher = torch.randn(n, V, generator=g, device="cuda").half()
    tids, tlp = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
    mp.mp_token_top(teacher if V % 8 == 0 else torch.nn.functional.pad(teacher, (0, -V % 8))[:, :V], tids, tlp, temperature=temp)
    w = torch.rand(n, generator=g, device="cuda") / n
    w[5:9] = 0
    model.distill_gradients(ids, tids, tlp, w, temp, tail)
    P = {name: t.double().requires_grad_() for name, t in model.w16.items()}
    loss = distill64(logits64(P, model, ids, lengths), tids, tlp, w.double(), temp, tail)
    grads = dict(zip(P, torch.autograd.grad(loss, list(P.values()))))
    assert abs(model.loss.item() - loss.item()) < 0.02 * abs(loss.item())
    for name, want in grads.items():
        got = model.dw[name].double() / 512.0
        off = (got - want).norm() / want.norm()
        # some 20 roundings of 2^-11 between the calls, on the way there and back
        assert off < 0.03, (name, off.item())
    h = model.state.read()
    assert h.found_inf == 0 and h.status == 0
    model.close()


def test_replayed_steps_follow_the_sequences(mp):
    """A recorded step of each kind equals eager ones bit for bit, also after the packing has changed."""
    from paper_1805_10387_b200.token_model import TokenModel
    n, V, k = 200, 61, 6
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    w = torch.full((n,), 1.0 / n, device="cuda")
    models = [TokenModel(V, 64, 128, 2, n, init_scale=256.0, state_bits=8, seed=5, heads=2, kv_heads=1, head_dim=64, sequences=3)
              for _ in range(2)]
    tids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:k] for _ in range(n)])
    tlp = torch.log_softmax(torch.randn(n, k + 1, generator=g, device="cuda"), 1)[:, :k].contiguous()
    args = (ids, tids, tlp, w)
    graph = models[0].capture(*args, step=models[0].distill_step)
    models[1].distill_step(*args)
    for lengths in ([200], [57, 143], [1, 0, 199]):
        for m in models:
            m.set_sequences(lengths)
        for _ in range(2):
            graph.replay()
            models[1].distill_step(*args)
    for name in models[0].w32:
        assert torch.equal(models[0].w32[name], models[1].w32[name]), name
    assert models[0].state.read().t == models[1].state.read().t == 7
    with pytest.raises(ValueError):
        models[0].set_sequences([100, 99])
    with pytest.raises(ValueError):
        models[0].set_sequences([50] * 4)
    for m in models:
        m.close()


def test_bad_offsets_freeze_the_step(mp):
    from paper_1805_10387_b200.token_model import TokenModel
    n, V = 300, 40
    model = TokenModel(V, 32, 64, 1, n, init_scale=64.0, heads=2, head_dim=32, sequences=3)
    ids = torch.arange(n, device="cuda") % V
    tids = (ids[:, None] + torch.arange(1, 4, device="cuda")) % V
    tlp, w = torch.full((n, 3), math.log(0.3), device="cuda"), torch.full((n,), 1.0 / n, device="cuda")
    model.distill_step(ids, tids, tlp, w)
    assert model.state.read().t == 1
    before = {name: t.clone() for name, t in model.w32.items()}
    for bad in ([0, 200, 100, 300], [0, 100, 200, 301], [-1, 100, 200, 300]):
        model.offsets.copy_(torch.tensor(bad, dtype=torch.int32))
        model.distill_step(ids, tids, tlp, w)
        h = model.state.read()
        assert h.status == mp.MP_ERR_INVALID_ARG and h.t == 1
        assert all(torch.equal(before[name], t) for name, t in model.w32.items())
        h.status, h.found_inf = 0, 0
        model.state.write(h)
    model.set_sequences([n])
    model.distill_step(ids, tids, tlp, w)
    assert model.state.read().t == 2
    model.close()


def test_the_demonstration_runs(mp):
    from paper_1805_10387_b200.token_model import demo, demo_distill
    _, _, teacher = demo(steps=2, tokens=500, keep=True)
    first, last = demo_distill(teacher, steps=3, length=128)
    assert math.isfinite(first) and math.isfinite(last)
    teacher.close()
