"""What is measured of the operators that let the token model mix tokens and learn from a teacher: their cases, inputs,
plain forms and 64-bit values.

Four operators: the norms of queries and keys for each head with the position rotation in the same pass, attention over
packed sequences with its backward pass, log-probabilities of given tokens with entropy and top alternatives, and
distillation from a teacher's top entries.  `run` computes a case with elementary torch operations in 32 bits (64 for the
angles of far positions), or, where `own` is set, with the calls that a user makes.
"""
import math
import random

import numpy as np
import torch

own = False

EPS, BASE, SCALE = 1e-6, 10000.0, 1024.0


def listed():
    return [
        # one new token for each of 16 sequences that are being generated: latency
        dict(name="heads_fwd_step", op="heads_fwd", T=16, hq=16, hk=4, D=64, rot=64, pairs=False, far=True),
        # a ragged batch, grouped heads, half of each head rotated in neighbouring pairs, positions far out
        dict(name="heads_fwd_ragged", op="heads_fwd", T=6387, hq=25, hk=5, D=128, rot=64, pairs=True, far=True),
        # the Transformer-like stack's rows, backward
        dict(name="heads_bwd_8192", op="heads_bwd", T=8192, hq=16, hk=16, D=64, rot=64, pairs=False, far=False),
        # one short sequence: latency
        dict(name="attn_fwd_short", op="attn_fwd", T=37, seqs=1, hq=16, hk=16, D=64, causal=True, window=0),
        # 64 x 400 frames of the speech stack, every frame sees its whole utterance
        dict(name="attn_fwd_frames", op="attn_fwd", T=25600, seqs=64, hq=25, hk=25, D=64, causal=False, window=0),
        # one long document, grouped heads
        dict(name="attn_fwd_long", op="attn_fwd", T=16384, seqs=1, hq=32, hk=8, D=128, causal=True, window=0),
        # a training batch of the Transformer-like stack: 16 sequences of uneven lengths
        dict(name="attn_bwd_8192", op="attn_bwd", T=8192, seqs=16, hq=16, hk=16, D=64, causal=True, window=0),
        # one long sequence, grouped heads, backward
        dict(name="attn_bwd_long", op="attn_bwd", T=8192, seqs=1, hq=16, hk=4, D=128, causal=True, window=0),
        # the 16 tokens that a step has just drawn, an odd and large vocabulary, many alternatives: latency
        dict(name="top_step", op="top", N=16, V=131071, k=64, temp=0.7, masked=0.0),
        # one batch of the Transformer-like stack with a subword output: the teacher's side of distillation
        dict(name="top_8192", op="top", N=8192, V=32768, k=20, temp=1.0, masked=0.1),
        # the student's side of it: the entries and everything else as one more outcome
        dict(name="distill_8192", op="distill", N=8192, V=32768, K=20, temp=1.0, tail=True, masked=0.1),
        # few rows of an odd, large vocabulary, many entries, softened
        dict(name="distill_wide", op="distill", N=1021, V=131071, K=128, temp=2.0, tail=False, masked=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["heads_fwd", "heads_bwd", "attn_fwd", "attn_bwd", "attn_fwd", "attn_bwd", "top", "distill"])
    if op.startswith("heads"):
        D = rng.choice([32, 64, 80, 128, 256])
        hk = rng.randint(1, 8)
        hq = hk * rng.choice([1, 2, 3, 4])
        return dict(op=op, T=_log(rng, 1, 40_000_000 // ((hq + hk) * D)), hq=hq, hk=hk, D=D, rot=rng.choice([16, D // 32 * 16, D]),
                    pairs=rng.random() < 0.5, far=rng.random() < 0.5)
    if op.startswith("attn"):
        D = rng.choice([32, 64, 72, 96, 128])
        hk = rng.choice([1, 2, 3, 4, 8])
        hq = hk * rng.choice([1, 2, 4])
        T = _log(rng, 1, 16384 if op == "attn_fwd" else 8192)
        window = _log(rng, 1, 2048) if rng.random() < 0.2 else 0
        return dict(op=op, T=T, seqs=_log(rng, 1, min(T, 64)), hq=min(hq, 16), hk=hk, D=D,
                    causal=window > 0 or rng.random() < 0.7, window=window)
    V = _log(rng, 200, 160_000)
    k, N = _log(rng, 1, 128), _log(rng, 1, min(40_000, 260_000_000 // V))
    masked, temp = rng.choice([0.0, 0.1, 0.5]), rng.choice([1.0, 0.6, 2.0])
    if op == "top":
        return dict(op=op, N=N, V=V, k=k, temp=temp, masked=masked)
    return dict(op=op, N=N, V=V, K=k, temp=temp, tail=rng.random() < 0.5, masked=masked)


# ---------------------------------------------------------------------------------------- inputs

def _up(n, a):
    return -(-n // a) * a


def _rows(g, rows, cols, std=1.0):
    """A [rows, cols] view of a buffer whose rows start on 16-byte boundaries, as the framework keeps them."""
    full = torch.zeros(rows, _up(cols, 8), dtype=torch.float16, device="cuda")
    full[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std
    return full[:, :cols]


def _empty(rows, cols):
    return torch.zeros(rows, _up(cols, 8), dtype=torch.float16, device="cuda")[:, :cols]


def _lengths(case):
    """Lengths of the packed sequences: uneven, some perhaps empty, T tokens in all (64 x 400 frames are even)."""
    T, B = case["T"], case["seqs"]
    if not case["causal"] and T % B == 0:
        return [T // B] * B
    raw = np.exp(0.7 * np.random.RandomState(T * 131 + B).randn(B))
    n = np.floor(raw / raw.sum() * T).astype(np.int64)
    n[0] += T - n.sum()
    return [int(x) for x in n]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = {"op": op, "case": case, "workspace": None}
    if op.startswith("heads"):
        T, hq, hk, D = (case[k] for k in ("T", "hq", "hk", "D"))
        # queries, keys and values of one product; the operator works on the first two
        s["qkv"] = _rows(g, T, (hq + 2 * hk) * D, std=1.5)
        s["x"] = s["qkv"][:, :(hq + hk) * D]
        start = torch.randint(0, 1_000_000 if case["far"] else 1, (1,), generator=g, device="cuda")
        s["pos"] = start + torch.arange(T, device="cuda") % 1000
        s["freqs"] = BASE ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        s["gq"], s["gk"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).half() for _ in range(2))
        if op == "heads_fwd":
            s["y"] = _empty(T, (hq + hk) * D)
        else:
            s["dy"] = _rows(g, T, (hq + hk) * D, std=0.5)
            s["dqkv"] = _empty(T, (hq + 2 * hk) * D)
            s["dx"] = s["dqkv"][:, :(hq + hk) * D]
            s["dgq"], s["dgk"] = (torch.zeros(D, dtype=torch.float16, device="cuda") for _ in range(2))
            if own:
                from paper_1805_10387_b200 import mp
                need = mp.mp_head_norm_rope_bwd_workspace_bytes(T, hq, hk, D)
                s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    elif op.startswith("attn"):
        T, hq, hk, D = (case[k] for k in ("T", "hq", "hk", "D"))
        s["lengths"] = _lengths(case)
        s["offsets"] = torch.tensor([0] + list(np.cumsum(s["lengths"])), dtype=torch.int32, device="cuda")
        qk = _rows(g, T, (hq + hk) * D)                      # normed and rotated queries and keys
        s["qkv"] = _rows(g, T, (hq + 2 * hk) * D)
        s["q"], s["k"], s["v"] = qk[:, :hq * D], qk[:, hq * D:], s["qkv"][:, (hq + hk) * D:]
        s["o"], s["lse"] = _empty(T, hq * D), torch.zeros(hq, T, device="cuda")
        if op == "attn_bwd":
            s["has_lse"] = False
            _plain_attn_fwd(s)
            s["has_lse"] = True
            s["do"] = _rows(g, T, hq * D, std=0.2)
            dqk = _empty(T, (hq + hk) * D)
            s["dq"], s["dk"], s["dv"] = dqk[:, :hq * D], dqk[:, hq * D:], _empty(T, (hq + 2 * hk) * D)[:, (hq + hk) * D:]
            if own:
                from paper_1805_10387_b200 import mp
                need = mp.mp_attention_bwd_workspace_bytes(T, hq, hk, D)
                s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    else:
        N, V = case["N"], case["V"]
        s["logits"] = _rows(g, N, V, std=2.0)
        live = torch.rand(N, generator=g, device="cuda") >= case["masked"]
        f32 = lambda *shape: torch.zeros(*shape, device="cuda")  # noqa: E731
        if op == "top":
            s["weight"] = live.float()
            s["targets"] = torch.randint(0, V, (N,), generator=g, device="cuda")
            s["logp"], s["entropy"], s["top_logp"] = f32(N), f32(N), f32(N, case["k"])
            s["top_ids"] = torch.zeros(N, case["k"], dtype=torch.int32, device="cuda")
        else:
            s["weight"] = live.float() / live.float().sum().clamp_(min=1)
            s["ids"], s["tlogp"] = (torch.empty(N, case["K"], dtype=t, device="cuda") for t in (torch.int32, torch.float32))
            for a in range(0, N, 1024):                      # a teacher that the student is some way from
                z = (s["logits"][a:a + 1024].float() + 0.7 * torch.randn(min(1024, N - a), V, generator=g, device="cuda")) / case["temp"]
                top = z.topk(case["K"], 1)
                s["ids"][a:a + 1024] = top.indices
                s["tlogp"][a:a + 1024] = top.values - torch.logsumexp(z, 1, keepdim=True)
            s["dlogits"], s["token_loss"], s["loss"] = _empty(N, V), f32(N), f32(1)
    return s


# ---------------------------------------------------------------------------------------- plain forms

def _pair(x, rot, pairs):
    """The two members of each rotated pair of columns."""
    if pairs:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _turn(x, pos, freqs, rot, pairs, back=False):
    """Rotates the pairs of x [T, heads, D] by pos * freqs (angles in 64 bits), in place."""
    a = pos.double()[:, None, None] * freqs
    c, s = a.cos().to(x.dtype), a.sin().to(x.dtype)
    if back:
        s = -s
    u, v = _pair(x, rot, pairs)
    nu, nv = u * c - v * s, u * s + v * c
    u.copy_(nu)
    v.copy_(nv)
    return x


def _gains(s, dtype):
    c = s["case"]
    return torch.cat([s["gq"].to(dtype).expand(c["hq"], -1), s["gk"].to(dtype).expand(c["hk"], -1)])[None]


def _plain_heads_fwd(s):
    c = s["case"]
    x = s["x"].float().view(c["T"], -1, c["D"])
    x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * _gains(s, x.dtype)
    s["y"].copy_(_turn(x, s["pos"], s["freqs"], c["rot"], c["pairs"]).view(c["T"], -1))
    return s["y"]


def _plain_heads_bwd(s):
    c = s["case"]
    x = s["x"].float().view(c["T"], -1, c["D"])
    u = _turn(s["dy"].float().view(c["T"], -1, c["D"]).clone(), s["pos"], s["freqs"], c["rot"], c["pairs"], back=True)
    root = torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)
    hat = x * root
    ug = u * hat
    s["dgq"].copy_(ug[:, :c["hq"]].sum((0, 1)))
    s["dgk"].copy_(ug[:, c["hq"]:].sum((0, 1)))
    d = u * _gains(s, x.dtype)
    s["dx"].copy_(((d - hat * (d * hat).mean(2, keepdim=True)) * root).view(c["T"], -1))
    return s["dx"], s["dgq"], s["dgk"]


def _hidden(n, causal, window):
    """True where query i does not see key j of the same sequence; None where every query sees every key."""
    if not causal:
        return None
    i = torch.arange(n, device="cuda")
    gap = i[:, None] - i[None, :]
    return (gap < 0) | (gap >= window) if window else gap < 0


def _parts(s):
    """(rows, key heads, mask) of one sequence and as many heads as there is room for scores."""
    c, at = s["case"], 0
    for n in s["lengths"]:
        if n:
            hidden = _hidden(n, c["causal"], c["window"])
            step = max(1, (1 << 28) // (n * n * (c["hq"] // c["hk"])))
            for h in range(0, c["hk"], step):
                yield slice(at, at + n), range(h, min(h + step, c["hk"])), hidden
        at += n


def _heads(t, rows, heads, D):
    """[heads, rows, D] of a matrix of rows, in 32 bits."""
    return t[rows, heads.start * D:heads.stop * D].float().view(-1, len(heads), D).transpose(0, 1)


def _grouped(s, name, rows, hs):
    """The rows of the query heads that share each key head, one below the other: [key heads, group * rows, D]."""
    c = s["case"]
    g = c["hq"] // c["hk"]
    return _heads(s[name], rows, range(hs.start * g, hs.stop * g), c["D"]).reshape(len(hs), -1, c["D"])


def _put(t, x, rows, heads, D):
    """Stores [.., rows, D] of the heads in their columns."""
    x = x.view(len(heads), -1, D).transpose(0, 1)
    t[rows, heads.start * D:heads.stop * D] = x.reshape(x.shape[0], -1).to(t.dtype)


def _probabilities(s, rows, hs, hidden):
    """exp(scores - row's largest) and that largest, or the probabilities where the row's log-sum is at hand."""
    c = s["case"]
    n, D, g = rows.stop - rows.start, c["D"], c["hq"] // c["hk"]
    x = (_grouped(s, "q", rows, hs) @ _heads(s["k"], rows, hs, D).transpose(1, 2)).mul_(D ** -0.5)
    if hidden is not None:
        x.view(-1, n, n).masked_fill_(hidden, -math.inf)
    if s["op"] == "attn_bwd" and s["has_lse"]:
        top = s["lse"][hs.start * g:hs.stop * g, rows].reshape(len(hs), -1, 1)
    else:
        top = x.amax(2, keepdim=True)
    return x.sub_(top).exp_(), top


def _plain_attn_fwd(s):
    c = s["case"]
    D, g = c["D"], c["hq"] // c["hk"]
    for rows, hs, hidden in _parts(s):
        p, top = _probabilities(s, rows, hs, hidden)
        total = p.sum(2, keepdim=True)
        qs = range(hs.start * g, hs.stop * g)
        _put(s["o"], (p @ _heads(s["v"], rows, hs, D)) / total, rows, qs, D)
        s["lse"][qs.start:qs.stop, rows] = (top + total.log()).view(len(qs), -1)
    return s["o"], s["lse"]


def _plain_attn_bwd(s):
    c = s["case"]
    D, g = c["D"], c["hq"] // c["hk"]
    for rows, hs, hidden in _parts(s):
        p, _ = _probabilities(s, rows, hs, hidden)
        do = _grouped(s, "do", rows, hs)
        delta = (do * _grouped(s, "o", rows, hs)).sum(2, keepdim=True)
        _put(s["dv"], p.transpose(1, 2) @ do, rows, hs, D)
        ds = (do @ _heads(s["v"], rows, hs, D).transpose(1, 2)).sub_(delta).mul_(p).mul_(D ** -0.5)
        _put(s["dk"], ds.transpose(1, 2) @ _grouped(s, "q", rows, hs), rows, hs, D)
        _put(s["dq"], ds @ _heads(s["k"], rows, hs, D), rows, range(hs.start * g, hs.stop * g), D)
    return s["dq"], s["dk"], s["dv"]


def _plain_top(s):
    c = s["case"]
    k = c["k"]
    for a in range(0, c["N"], 2048):                         # a block of rows at a time, for the sort's room
        b = slice(a, min(a + 2048, c["N"]))
        z = s["logits"][b].float() / c["temp"]
        live = s["weight"][b] != 0
        top, order = s["logits"][b].sort(dim=1, descending=True, stable=True)     # ties: the lowest index first
        z -= z.amax(1, keepdim=True)
        total = z.exp().sum(1, keepdim=True)
        lp = z - total.log()
        s["logp"][b] = torch.where(live, lp.gather(1, s["targets"][b][:, None])[:, 0], 0.0)
        s["entropy"][b] = torch.where(live, -(lp.exp() * lp).sum(1), 0.0)
        s["top_ids"][b] = torch.where(live[:, None], order[:, :k], -1).int()
        s["top_logp"][b] = torch.where(live[:, None], lp.gather(1, order[:, :k]), 0.0)
    return s["logp"], s["entropy"], s["top_ids"], s["top_logp"]


def _plain_distill(s):
    c, w = s["case"], s["weight"]
    ids, a = s["ids"].long(), s["tlogp"]
    z = s["logits"].float() / c["temp"]
    z -= z.amax(1, keepdim=True)
    zt = z.gather(1, ids)
    e = z.exp_()
    total = e.sum(1, keepdim=True)
    lq = zt - total.log()
    if c["tail"]:
        p = a.exp()
        e.scatter_(1, ids, 0.0)
        rest = e.sum(1, keepdim=True)                        # of what the teacher does not list
        pr = (1 - p.sum(1, keepdim=True)).clamp_(min=0)
        tail = torch.where(pr > 0, pr * (pr.log() - (rest / total).log()), 0.0)
        loss = (p * (a - lq)).sum(1) + tail[:, 0]
        grad = e.mul_(1 / total - pr / rest)
    else:
        a = a - torch.logsumexp(a, 1, keepdim=True)
        p = a.exp()
        loss = (p * (a - lq)).sum(1)
        grad = e.div_(total)
    grad.scatter_(1, ids, lq.exp() - p)
    grad *= (SCALE / c["temp"] * w)[:, None]
    s["dlogits"].copy_(grad)
    s["token_loss"].copy_(w * loss)
    s["loss"].copy_(s["token_loss"].sum())
    return s["dlogits"], s["token_loss"], s["loss"]


# ---------------------------------------------------------------------------------------- a pass

def _own(s):
    from paper_1805_10387_b200 import mp
    op, c = s["op"], s["case"]
    if op == "heads_fwd":
        mp.mp_head_norm_rope_fwd(s["x"], s["gq"], s["gk"], s["pos"], s["freqs"], s["y"], c["hq"], c["hk"], eps=EPS,
                                 pairs=c["pairs"])
        return s["y"]
    if op == "heads_bwd":
        mp.mp_head_norm_rope_bwd(s["dy"], s["x"], s["gq"], s["gk"], s["pos"], s["freqs"], s["dx"], s["dgq"], s["dgk"],
                                 c["hq"], c["hk"], eps=EPS, pairs=c["pairs"], workspace=s["workspace"])
        return s["dx"], s["dgq"], s["dgk"]
    if op == "attn_fwd":
        mp.mp_attention_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["offsets"], c["hq"], c["hk"], causal=c["causal"],
                            window=c["window"])
        return s["o"], s["lse"]
    if op == "attn_bwd":
        mp.mp_attention_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"], s["offsets"],
                            c["hq"], c["hk"], causal=c["causal"], window=c["window"], workspace=s["workspace"])
        return s["dq"], s["dk"], s["dv"]
    if op == "top":
        mp.mp_token_top(s["logits"], s["top_ids"], s["top_logp"], targets=s["targets"], logp=s["logp"], entropy=s["entropy"],
                        weight=s["weight"], temperature=c["temp"])
        return s["logp"], s["entropy"], s["top_ids"], s["top_logp"]
    mp.mp_distill_loss(s["logits"], s["ids"], s["tlogp"], s["weight"], s["token_loss"], loss=s["loss"], dlogits16=s["dlogits"],
                       temperature=c["temp"], tail=c["tail"], grad_scale=SCALE)
    return s["dlogits"], s["token_loss"], s["loss"]


def run(state):
    if own:
        return _own(state)
    return {"heads_fwd": _plain_heads_fwd, "heads_bwd": _plain_heads_bwd, "attn_fwd": _plain_attn_fwd, "attn_bwd": _plain_attn_bwd,
            "top": _plain_top, "distill": _plain_distill}[state["op"]](state)


def _seen(case):
    """Pairs of a query and a key that it sees."""
    total = 0
    for n in _lengths(case):
        w = min(case["window"] or n, n)
        total += n * w - w * (w - 1) // 2 if case["causal"] else n * n
    return total


def work(case):
    op = case["op"]
    if op.startswith("heads"):
        n = case["T"] * (case["hq"] + case["hk"]) * case["D"]
        fwd = op == "heads_fwd"
        return {"bytes": n * (4 if fwd else 6) + case["T"] * 8 + case["D"] * (4 if fwd else 8), "flops": n * (7 if fwd else 14)}
    if op.startswith("attn"):
        T, D, hq, hk = case["T"], case["D"], case["hq"], case["hk"]
        if op == "attn_fwd":
            return {"bytes": 4 * T * D * (hq + hk) + 4 * T * hq, "flops": 4 * D * hq * _seen(case)}
        return {"bytes": 2 * T * D * (4 * hq + 4 * hk) + 4 * T * hq, "flops": 10 * D * hq * _seen(case)}
    N, V, live = case["N"], case["V"], case["N"] * (1 - case["masked"])
    if op == "top":
        return {"bytes": 2 * V * live + N * (20 + 8 * case["k"]), "flops": 6 * live * V}
    return {"bytes": 2 * V * (live + N) + N * (8 + 8 * case["K"]), "flops": 6 * live * V}


# ---------------------------------------------------------------------------------------- 64 bits

def _rotated(x, s):
    """x times exp(i pos freq) on the pairs as complex numbers."""
    c = s["case"]
    rot = c["rot"]
    turn = torch.exp(1j * (s["pos"].double()[:, None, None] * s["freqs"]))
    u, v = _pair(x, rot, c["pairs"])
    w = torch.complex(u, v) * turn
    if c["pairs"]:
        turned = torch.stack([w.real, w.imag], 3).flatten(2)
    else:
        turned = torch.cat([w.real, w.imag], 2)
    return torch.cat([turned, x[..., rot:]], 2)


def _exact_heads(x, gq, gk, s):
    c = s["case"]
    x = x.view(c["T"], -1, c["D"])
    norm = x / torch.sqrt((x * x).mean(2, keepdim=True) + EPS)
    return _rotated(torch.cat([norm[:, :c["hq"]] * gq, norm[:, c["hq"]:] * gk], 1), s).reshape(c["T"], -1)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = lambda k: s[k].double()  # noqa: E731
    leaf = lambda k: d(k).requires_grad_()  # noqa: E731
    if op == "heads_fwd":
        return _exact_heads(d("x"), d("gq"), d("gk"), s)
    if op == "heads_bwd":
        x, gq, gk = leaf("x"), leaf("gq"), leaf("gk")
        return torch.autograd.grad(_exact_heads(x, gq, gk, s), (x, gq, gk), d("dy"))
    if op.startswith("attn"):
        D, hq, hk = case["D"], case["hq"], case["hk"]
        back = op == "attn_bwd"
        out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in (("dq", "dk", "dv") if back else ("o", "lse"))}
        at = 0
        for n in s["lengths"]:
            r = slice(at, at + n)
            at += n
            for h in range(hq if n else 0):
                a, b = slice(h * D, (h + 1) * D), slice(h * hk // hq * D, (h * hk // hq + 1) * D)
                q, k, v = s["q"][r, a].double(), s["k"][r, b].double(), s["v"][r, b].double()
                x = torch.einsum("id,jd->ij", q, k) / math.sqrt(D)
                if case["causal"]:
                    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril_()
                    if case["window"]:
                        seen.triu_(1 - case["window"])
                    x = torch.where(seen, x, -math.inf)
                    del seen
                if not back:
                    out["lse"][h, r] = torch.logsumexp(x, 1)
                    out["o"][r, a] = torch.softmax(x, 1) @ v
                    continue
                p, do = torch.softmax(x, 1), s["do"][r, a].double()
                out["dv"][r, b] += p.T @ do
                g = do @ v.T
                x = p * (g - (p * g).sum(1, keepdim=True)) / math.sqrt(D)
                out["dq"][r, a] = x @ k
                out["dk"][r, b] += x.T @ q
        return tuple(out.values())
    live = s["weight"] != 0
    outs = []
    for a in range(0, case["N"], 1024):                      # rows do not depend on one another
        b = slice(a, a + 1024)
        z, on = s["logits"][b].double() / case["temp"], live[b]
        if op == "top":
            lp = torch.log_softmax(z, 1)
            # order of the values, then of the indices, as one whole number
            bits = (s["logits"][b] + 0.0).view(torch.int16).long()
            key = torch.where(bits < 0, -(bits & 0x7FFF), bits) * (1 << 20) - torch.arange(case["V"], device="cuda")
            ids = key.topk(case["k"], 1).indices
            outs.append((torch.where(on, lp.gather(1, s["targets"][b][:, None])[:, 0], 0.0),
                         torch.where(on, torch.distributions.Categorical(logits=z).entropy(), 0.0),
                         torch.where(on[:, None], ids, -1).int(), torch.where(on[:, None], lp.gather(1, ids), 0.0)))
            continue
        z.requires_grad_()
        ids, t = s["ids"][b].long(), s["tlogp"][b].double()
        lq = torch.log_softmax(z, 1)
        if case["tail"]:
            other = torch.ones_like(z, dtype=torch.bool).scatter_(1, ids, False)
            lr = torch.logsumexp(torch.where(other, lq, -math.inf), 1)
            p = t.exp()
            pr = 1 - p.sum(1)
            loss = (p * (t - lq.gather(1, ids))).sum(1) + torch.where(pr > 0, pr * (pr.clamp(min=1e-300).log() - lr), 0.0)
        else:
            t = torch.log_softmax(t, 1)
            loss = (t.exp() * (t - lq.gather(1, ids))).sum(1)
        loss = torch.where(on, s["weight"][b].double() * loss, 0.0)
        (grad,) = torch.autograd.grad(loss.sum() * SCALE, z)
        outs.append((grad / case["temp"], loss.detach()))
    cols = tuple(torch.cat(c) for c in zip(*outs))
    return cols if op == "top" else cols + (cols[1].sum()[None],)


if __name__ == "__main__":
    r = random.Random(0)
    for c in listed() + [draw(r) for _ in range(6)]:
        print(c, work(c))
