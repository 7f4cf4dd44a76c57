"""What is measured of the token-model operators: their cases, inputs, plain forms and 64-bit values.

Four operators around the products of a training step: the embedding lookup and its gradient, the norms
before and after a block with its gate and residual scale, the clipped policy loss with a KL term, and AdamW
over many tensors with states in 32 or in 8 bits.  `run` computes a case with elementary torch operations in
32 bits, or, where `own` is set, with the calls that a user makes.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 256          # elements that share one scale in the 8-bit states
LR, BETA1, BETA2, EPS, DECAY, SCALE, T0 = 1e-3, 0.9, 0.95, 1e-8, 0.1, 1024.0, 100
CLIP_LO, CLIP_HI, KL = 0.2, 0.28, 0.05
NORM_EPS = 1e-6


def listed():
    return [
        # one new token for each of 16 sequences that are being generated: latency
        dict(name="embed_fwd_step", op="embed_fwd", n=16, V=32768, D=1024, wide_ids=True),
        # gradient of a subword table over one batch of the Transformer-like stack
        dict(name="embed_bwd_subwords", op="embed_bwd", n=8192, V=32768, D=1024, wide_ids=True),
        # gradient of a 29-symbol table over 64 x 400 frames: few rows, each summed over hundreds of tokens
        dict(name="embed_bwd_symbols", op="embed_bwd", n=25600, V=29, D=1600, wide_ids=False),
        # one new token for each of 16 sequences through the norms of a block: latency
        dict(name="norm_fwd_step", op="norm_fwd", M=16, D=1024, layer=False, wide=False, gate="shared", res=1.0),
        # the Transformer-like stack's rows, forward
        dict(name="norm_fwd_8192", op="norm_fwd", M=8192, D=1024, layer=False, wide=False, gate="shared", res=1.0),
        # a ragged batch of odd width, mean and variance, FP32 residual stream, a gate for every token
        dict(name="norm_bwd_ragged", op="norm_bwd", M=6387, D=1001, layer=True, wide=True, gate="token", res=0.7),
        # the speech stack's rows, backward
        dict(name="norm_bwd_25600", op="norm_bwd", M=25600, D=1600, layer=False, wide=False, gate="shared", res=1.0),
        # a 29-symbol output over 64 x 400 frames: many short rows
        dict(name="loss_symbols", op="loss", N=25600, V=29, kl=True, masked=0.1),
        # one batch of the Transformer-like stack with a subword output: the ordinary case
        dict(name="loss_8192", op="loss", N=8192, V=32768, kl=True, masked=0.1),
        # an odd, large vocabulary and few rows: a row no longer fits one block's registers
        dict(name="loss_wide_vocab", op="loss", N=1021, V=131071, kl=False, masked=0.3),
        # the parameters of a small model, 32-bit states
        dict(name="adamw32_1e7", op="adamw", P=10_000_000, tensors=50, bits=32),
        # 1e8 parameters in 500 tensors of log-uniform sizes, 8-bit states
        dict(name="adamw8_1e8", op="adamw", P=100_000_000, tensors=500, bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "loss", "adamw"])
    if op.startswith("embed"):
        D = _log(rng, 64, 4096)
        return dict(op=op, n=_log(rng, 1, min(65536, 41_000_000 // D)), V=_log(rng, 29, min(65536, 67_000_000 // D)), D=D,
                    wide_ids=rng.random() < 0.5)
    if op.startswith("norm"):
        D = _log(rng, 64, 8192)
        return dict(op=op, M=_log(rng, 1, 40_000_000 // D), D=D, layer=rng.random() < 0.5, wide=rng.random() < 0.5,
                    gate=rng.choice(["none", "shared", "token"]), res=rng.choice([1.0, 0.7]))
    if op == "loss":
        V = _log(rng, 29, 160_000)
        return dict(op=op, N=_log(rng, 16, min(40_000, 260_000_000 // V)), V=V, kl=rng.random() < 0.5,
                    masked=rng.choice([0.0, 0.1, 0.5]))
    return dict(op=op, P=_log(rng, 100_000, 100_000_000), tensors=_log(rng, 1, 500), bits=rng.choice([8, 32]))


# ---------------------------------------------------------------------------------------- inputs

def _up(n, a):
    return -(-n // a) * a


def _rows(g, rows, cols, dtype=torch.float16, std=1.0, mean=0.0):
    """A [rows, cols] view of a buffer whose rows start on 16-byte boundaries, as the framework keeps them."""
    full = torch.zeros(rows, _up(cols, 8), dtype=dtype, device="cuda")
    full[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std + mean
    return full[:, :cols]


def _empty(rows, cols, dtype=torch.float16):
    return torch.zeros(rows, _up(cols, 8), dtype=dtype, device="cuda")[:, :cols]


def _zipf(g, n, V):
    """Tokens whose frequency falls as 1 / rank; token 0 is the padding of the tails of sequences."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V)) - 1).long().clamp_(0, V - 1)
    return torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, 0, ids)


def _sizes(P, tensors):
    """The sizes of a model's tensors: log-uniform over four decades, about P in all."""
    r = np.random.RandomState(tensors)
    raw = np.exp(r.rand(tensors) * math.log(1e4))
    return np.maximum(1, np.floor(raw / raw.sum() * P)).astype(np.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = {"op": op, "case": case}
    if op.startswith("embed"):
        n, V, D = case["n"], case["V"], case["D"]
        s["ids"] = _zipf(g, n, V).to(torch.int64 if case["wide_ids"] else torch.int32)
        s["scale"] = math.sqrt(D)
        if op == "embed_fwd":
            s["w"], s["y"] = _rows(g, V, D, std=D ** -0.5), _empty(n, D)
        else:
            s["dy"], s["dw"] = _rows(g, n, D, std=0.05), _empty(V, D)
            s["workspace"] = None
    elif op.startswith("norm"):
        M, D = case["M"], case["D"]
        xt = torch.float32 if case["wide"] else torch.float16
        s["y"] = _rows(g, M, D, std=2.0, mean=0.2)
        s["g_post"], s["g_pre"] = (_rows(g, 1, D, std=0.1, mean=1.0)[0] for _ in range(2))
        s["gate"] = None if case["gate"] == "none" else _rows(g, 1, D, std=0.3, mean=0.5)[0] if case["gate"] == "shared" \
            else _rows(g, M, D, std=0.3, mean=0.5)
        if op == "norm_fwd":
            s["x"] = _rows(g, M, D, xt, std=3.0, mean=0.3)
            s["x_out"], s["n"] = _empty(M, D, xt), _empty(M, D)
            s["stats"] = torch.zeros(M, 4, device="cuda")
        else:
            s["x_out"] = _rows(g, M, D, xt, std=3.0, mean=0.3)
            s["dn"], s["dx_out"] = _rows(g, M, D, std=0.5), _rows(g, M, D, xt, std=0.5)
            s["stats"] = torch.cat([_stats(s["y"].float(), case["layer"]), _stats(s["x_out"].float(), case["layer"])], 1)
            s["dx"], s["dy"] = _empty(M, D, xt), _empty(M, D)
            s["dg_post"], s["dg_pre"] = (_empty(1, D)[0] for _ in range(2))
            s["dgate"] = None if case["gate"] == "none" else _empty(1, D)[0] if case["gate"] == "shared" else _empty(M, D)
            s["workspace"] = None
    elif op == "loss":
        N, V = case["N"], case["V"]
        s["logits"], s["dlogits"] = _rows(g, N, V, std=2.0), _empty(N, V)
        s["targets"] = _zipf(g, N, V)
        z = s["logits"].float()
        lp = z.gather(1, s["targets"][:, None])[:, 0] - torch.logsumexp(z, 1)
        del z
        jitter = lambda std: std * torch.randn(N, generator=g, device="cuda")  # noqa: E731
        s["old"] = lp + jitter(0.15)
        s["ref"] = lp + jitter(0.3) if case["kl"] else None
        s["adv"] = 0.5 + jitter(1.0)
        live = (torch.rand(N, generator=g, device="cuda") >= case["masked"]).float()
        s["weight"] = live / live.sum().clamp_(min=1)
        s["logp"], s["token_loss"], s["loss"] = (torch.zeros(k, device="cuda") for k in (N, N, 1))
    else:
        counts = _sizes(case["P"], case["tensors"])
        starts = np.concatenate([[0], np.cumsum(_up(counts, BLOCK))])
        total = int(starts[-1])
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        at = [slice(int(a), int(a + c)) for a, c in zip(starts, counts)]
        for k in at:
            live[k] = True
        z = lambda: torch.randn(total, generator=g, device="cuda") * live  # noqa: E731
        s["g"] = (z() * 1e-3 * SCALE).half()
        s["w"] = z() * 0.02
        s["w16"] = s["w"].half()
        m, r = z() * 3e-4, (z() * 2e-4).abs() + 8e-4 * live
        s["decay"] = np.where(np.random.RandomState(seed % (1 << 31)).rand(len(counts)) < 0.7, 1.0, 0.0).astype(np.float32)
        s["decay_of_block"] = torch.from_numpy(np.repeat(s["decay"], _up(counts, BLOCK) // BLOCK)).cuda()
        s["t"], s["m_scale"], s["v_scale"] = T0, None, None
        if case["bits"] == 32:
            s["m"], s["v"] = m, r * r
        else:
            s["m"], s["m_scale"] = _quantise(m, False)
            s["v"], s["v_scale"] = _quantise(r, True)
        if own:          # the handles that a training program keeps: the loss-scale state and the update's plan
            from paper_1805_10387_b200 import mp
            s["state"] = mp.State(SCALE, dynamic=False)
            h = s["state"].read()
            h.t = T0
            s["state"].write(h)
            cut = lambda t: [t[k] for k in at]  # noqa: E731
            cut_s = lambda t: None if t is None else [t[k.start // BLOCK:-(-k.stop // BLOCK)] for k in at]  # noqa: E731
            s["plan"] = mp.AdamWPlan(cut(s["g"]), cut(s["w"]), cut(s["m"]), cut(s["v"]), cut(s["w16"]),
                                     m_scale=cut_s(s["m_scale"]), v_scale=cut_s(s["v_scale"]), decay=s["decay"].tolist())
            s["opt"] = mp.AdamWConfig(LR, BETA1, BETA2, EPS, DECAY)
    if own and op in ("embed_bwd", "norm_bwd"):      # the scratch that a training program keeps for its calls
        from paper_1805_10387_b200 import mp
        need = mp.mp_embedding_bwd_workspace_bytes(case["n"], case["V"], case["D"]) if op == "embed_bwd" \
            else mp.mp_block_norm_bwd_workspace_bytes(case["M"], case["D"])
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------- plain forms

def _stats(v, layer):
    """[mean, 1 / root] of each row; the mean is 0 for the root-mean-square norm."""
    mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    return torch.cat([mean, torch.rsqrt((v - mean).square().mean(1, keepdim=True) + NORM_EPS)], 1)


def _norm_bwd(d, hat, root, layer):
    """Gradient at v of sum(d * hat), hat = (v - mean) * root."""
    out = d - hat * (d * hat).mean(1, keepdim=True)
    if layer:
        out = out - d.mean(1, keepdim=True)
    return out * root


def _quantise(v, keep):
    """E4M3 numbers and one scale for each BLOCK elements; `keep`: what is above zero does not become zero."""
    b = v.view(-1, BLOCK)
    top = b.abs().amax(1)
    inv = torch.where(top > 0, 448.0 / top, 0.0)
    q = b * inv[:, None]
    if keep:
        q = torch.where(b > 0, q.clamp(min=2.0 ** -9), q)
    return q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(-1), top / 448.0


def _plain_embed_fwd(s):
    y = s["w"].index_select(0, s["ids"]).float() * s["scale"]
    s["y"].copy_(y.masked_fill_((s["ids"] == 0)[:, None], 0.0))
    return s["y"]


def _plain_embed_bwd(s):
    acc = torch.zeros(s["dw"].shape, device="cuda")
    acc.index_add_(0, s["ids"], s["dy"].float().masked_fill_((s["ids"] == 0)[:, None], 0.0))
    s["dw"].copy_(acc * s["scale"])
    return s["dw"]


def _plain_norm_fwd(s):
    c, y, x = s["case"], s["y"].float(), s["x"].float()
    ys = _stats(y, c["layer"])
    h = (y - ys[:, :1]) * ys[:, 1:] * s["g_post"].float()
    if s["gate"] is not None:
        h = h * s["gate"].float()
    x = c["res"] * x + h
    xs = _stats(x, c["layer"])
    s["n"].copy_((x - xs[:, :1]) * xs[:, 1:] * s["g_pre"].float())
    s["x_out"].copy_(x)
    s["stats"][:, :2] = ys
    s["stats"][:, 2:] = xs
    return s["x_out"], s["n"], s["stats"]


def _plain_norm_bwd(s):
    c, st, dn = s["case"], s["stats"], s["dn"].float()
    xhat = (s["x_out"].float() - st[:, 2:3]) * st[:, 3:4]
    yhat = (s["y"].float() - st[:, 0:1]) * st[:, 1:2]
    gx = s["dx_out"].float() + _norm_bwd(dn * s["g_pre"].float(), xhat, st[:, 3:4], c["layer"])
    s["dx"].copy_(c["res"] * gx)
    s["dg_pre"].copy_((dn * xhat).sum(0))
    dh = gx
    if s["gate"] is not None:
        dgate = gx * yhat * s["g_post"].float()
        s["dgate"].copy_(dgate.sum(0) if c["gate"] == "shared" else dgate)
        dh = gx * s["gate"].float()
    s["dg_post"].copy_((dh * yhat).sum(0))
    s["dy"].copy_(_norm_bwd(dh * s["g_post"].float(), yhat, st[:, 1:2], c["layer"]))
    return s["dx"], s["dy"], s["dg_pre"], s["dg_post"], s["dgate"]


def _plain_loss(s):
    z = s["logits"].float()
    z -= z.amax(1, keepdim=True)
    zt = z.gather(1, s["targets"][:, None])
    p = z.exp_()
    total = p.sum(1, keepdim=True)
    p /= total
    w = s["weight"]
    live = w != 0
    lp = torch.where(live, (zt - total.log())[:, 0], 0.0)
    r = torch.exp(lp - s["old"])
    a = r * s["adv"]
    b = r.clamp(1 - CLIP_LO, 1 + CLIP_HI) * s["adv"]
    loss, d = -torch.minimum(a, b), torch.where(a <= b, -a, 0.0)
    if s["ref"] is not None:
        e = s["ref"] - lp
        loss = loss + KL * (torch.expm1(e) - e)
        d = d - KL * torch.expm1(e)
    s["logp"].copy_(lp)
    s["token_loss"].copy_(torch.where(live, w * loss, 0.0))
    s["loss"].copy_(s["token_loss"].sum())
    d = torch.where(live, SCALE * w * d, 0.0)[:, None]
    p.neg_().scatter_add_(1, s["targets"][:, None], torch.ones_like(d))
    p *= d
    s["dlogits"].copy_(p)
    return s["dlogits"], s["logp"], s["token_loss"], s["loss"]


def _plain_adamw(s):
    s["t"] += 1
    c1, c2 = 1 - BETA1 ** s["t"], 1 - BETA2 ** s["t"]
    g = s["g"].float() * (1 / SCALE)
    wide = s["case"]["bits"] == 32
    if wide:
        m, v = s["m"], s["v"]
    else:
        value = lambda q, scale: (q.float().view(-1, BLOCK) * scale[:, None]).view(-1)  # noqa: E731
        m, v = value(s["m"], s["m_scale"]), value(s["v"], s["v_scale"]).square_()
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g.square_() * (1 - BETA2))
    r = v.sqrt()
    w = s["w"].view(-1, BLOCK)
    w -= w * (LR * DECAY * s["decay_of_block"])[:, None]
    s["w"] -= (LR / c1) * (m / (r * (1 / math.sqrt(c2)) + EPS))
    s["w16"].copy_(s["w"])
    if not wide:
        s["m"], s["m_scale"] = _quantise(m, False)
        s["v"], s["v_scale"] = _quantise(r, True)
    return s["w"], s["w16"], s["m"], s["v"], s["m_scale"], s["v_scale"]


# ---------------------------------------------------------------------------------------- a pass

def _own(s):
    from paper_1805_10387_b200 import mp
    op, c = s["op"], s["case"]
    if op == "embed_fwd":
        mp.mp_embedding_fwd(s["ids"], s["w"], s["y"], pad_id=0, scale=s["scale"])
        return s["y"]
    if op == "embed_bwd":
        mp.mp_embedding_bwd(s["ids"], s["dy"], s["dw"], pad_id=0, scale=s["scale"], workspace=s["workspace"])
        return s["dw"]
    if op == "norm_fwd":
        mp.mp_block_norm_fwd(s["x"], s["g_pre"], s["n"], s["stats"], y16=s["y"], g_post16=s["g_post"], gate16=s["gate"],
                             x_out=s["x_out"], kind=mp.MP_NORM_LAYER if c["layer"] else mp.MP_NORM_RMS, eps=NORM_EPS,
                             res_scale=c["res"])
        return s["x_out"], s["n"], s["stats"]
    if op == "norm_bwd":
        mp.mp_block_norm_bwd(s["dn"], s["x_out"], s["g_pre"], s["stats"], s["dx"], s["dg_pre"], dx_out=s["dx_out"],
                             y16=s["y"], g_post16=s["g_post"], gate16=s["gate"], dy16=s["dy"], dg_post16=s["dg_post"],
                             dgate16=s["dgate"], kind=mp.MP_NORM_LAYER if c["layer"] else mp.MP_NORM_RMS,
                             res_scale=c["res"], workspace=s["workspace"])
        return s["dx"], s["dy"], s["dg_pre"], s["dg_post"], s["dgate"]
    if op == "loss":
        mp.mp_policy_loss(s["logits"], s["targets"], s["old"], s["adv"], s["weight"], s["logp"], s["token_loss"],
                          s["loss"], dlogits16=s["dlogits"], ref_logp=s["ref"], clip_lo=CLIP_LO, clip_hi=CLIP_HI,
                          kl_coef=KL if s["ref"] is not None else 0.0, grad_scale=SCALE)
        return s["dlogits"], s["logp"], s["token_loss"], s["loss"]
    mp.mp_adamw_update(s["plan"], s["state"], s["opt"])
    mp.mp_loss_scale_update(s["state"])
    return s["w"], s["w16"], s["m"], s["v"], s["m_scale"], s["v_scale"]


def run(state):
    if own:
        return _own(state)
    return {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd, "norm_fwd": _plain_norm_fwd,
            "norm_bwd": _plain_norm_bwd, "loss": _plain_loss, "adamw": _plain_adamw}[state["op"]](state)


def work(case):
    op = case["op"]
    if op.startswith("embed"):
        n, V, D = case["n"], case["V"], case["D"]
        table = min(n, V) if op == "embed_fwd" else V
        return {"bytes": n * (8 if case["wide_ids"] else 4) + 2 * D * (n + table), "flops": n * D}
    if op.startswith("norm"):
        M, D, x = case["M"], case["D"], 4 if case["wide"] else 2
        gate = {"none": 0, "shared": 2 * D, "token": 2 * M * D}[case["gate"]]
        if op == "norm_fwd":
            return {"bytes": M * D * (2 * x + 4) + gate + 4 * D + 16 * M, "flops": 14 * M * D}
        return {"bytes": M * D * (3 * x + 6) + 2 * gate + 8 * D + 16 * M, "flops": 26 * M * D}
    if op == "loss":
        N, V = case["N"], case["V"]
        live = N * (1 - case["masked"])
        return {"bytes": 2 * V * (live + N) + N * (8 + 4 * (6 if case["kl"] else 5)), "flops": 6 * live * V}
    return {"bytes": case["P"] * (28 if case["bits"] == 32 else 16 + 16 / BLOCK), "flops": 20 * case["P"]}


# ---------------------------------------------------------------------------------------- 64 bits

def _exact_norm(v, gain, layer):
    if layer:
        v = v - v.mean(1, keepdim=True)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + NORM_EPS) * gain


def _exact_e4m3(v, keep):
    """E4M3 by its definition: three bits of fraction above 2^-6, steps of 2^-9 below; ties to the even step."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.round(v / step) * step
    return torch.where((v > 0) & (q == 0), 2.0 ** -9, q) if keep else q


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = lambda k: None if s[k] is None else s[k].double()  # noqa: E731
    if op.startswith("embed"):
        kept = (s["ids"] != 0).nonzero()[:, 0]
        ids = s["ids"].long()[kept]
        if op == "embed_fwd":
            y = torch.zeros(case["n"], case["D"], dtype=torch.float64, device="cuda")
            y[kept] = d("w")[ids] * math.sqrt(case["D"])
            return y
        order = torch.argsort(ids, stable=True)
        dw = torch.zeros(case["V"], case["D"], dtype=torch.float64, device="cuda")
        return dw.index_put_((ids[order],), d("dy")[kept[order]] * math.sqrt(case["D"]), accumulate=True)
    if op == "norm_fwd":
        gate = 1.0 if s["gate"] is None else d("gate")
        x = case["res"] * d("x") + gate * _exact_norm(d("y"), d("g_post"), case["layer"])
        moments = []
        for v in (d("y"), x):
            mean = v.mean(1) if case["layer"] else torch.zeros_like(v[:, 0])
            moments += [mean, 1 / torch.sqrt(((v - mean[:, None]) ** 2).mean(1) + NORM_EPS)]
        return x, _exact_norm(x, d("g_pre"), case["layer"]), torch.stack(moments, 1)
    if op == "norm_bwd":
        leaf = lambda k: d(k).requires_grad_()  # noqa: E731
        x, gp = leaf("x_out"), leaf("g_pre")
        gx, dg_pre = torch.autograd.grad(_exact_norm(x, gp, case["layer"]), (x, gp), d("dn"))
        gx = gx + d("dx_out")
        y, go = leaf("y"), leaf("g_post")
        h = _exact_norm(y, go, case["layer"])
        if s["gate"] is None:
            dy, dg_post = torch.autograd.grad(h, (y, go), gx)
            return case["res"] * gx, dy, dg_pre, dg_post, None
        gate = leaf("gate")
        dy, dg_post, dgate = torch.autograd.grad(h * gate, (y, go, gate), gx)
        return case["res"] * gx, dy, dg_pre, dg_post, dgate
    if op == "loss":
        z = d("logits").requires_grad_()
        live = s["weight"] != 0
        lp = torch.log_softmax(z, 1).gather(1, s["targets"][:, None])[:, 0]
        surrogate, ratio = d("adv") * torch.exp(lp - d("old")), torch.exp(lp - d("old"))
        clipped = torch.clamp(ratio, 1 - CLIP_LO, 1 + CLIP_HI) * d("adv")
        loss = -torch.where(surrogate <= clipped, surrogate, clipped)
        if s["ref"] is not None:
            gap = d("ref") - lp
            loss = loss + KL * (torch.exp(gap) - gap - 1)
        loss = torch.where(live, d("weight") * loss, 0.0)
        (grad,) = torch.autograd.grad(loss.sum() * SCALE, z)
        return grad, torch.where(live, lp, 0.0).detach(), loss.detach(), loss.sum().detach()[None]
    t = T0 + 1
    g = d("g") / SCALE
    wide = case["bits"] == 32
    spread = lambda k: d(k).repeat_interleave(BLOCK)  # noqa: E731
    m = d("m") if wide else d("m") * spread("m_scale")
    v = d("v") if wide else (d("v") * spread("v_scale")) ** 2
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
    w = d("w") * (1 - LR * DECAY * spread("decay_of_block"))
    w = w - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    if wide:
        return w, w, m, v, None, None
    kept = []
    for x, keep in ((m, False), (torch.sqrt(v), True)):
        top = x.view(-1, BLOCK).abs().amax(1) / 448
        kept.append((_exact_e4m3(x / top.clamp(min=1e-300).repeat_interleave(BLOCK), keep), top))
    return w, w, kept[0][0], kept[1][0], kept[0][1], kept[1][1]


if __name__ == "__main__":
    r = random.Random(0)
    for c in listed() + [draw(r) for _ in range(6)]:
        print(c, work(c))
