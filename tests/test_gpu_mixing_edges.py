"""Edges of attention, head norms, token scores and distillation: recorded and concurrent calls, many and far rows, values of other
sequences, scaled gradients, differences, many rows for each worker."""
import math

import pytest
import torch

from test_gpu_attention import Case, H
from test_gpu_head_norm import Case as HeadCase
from test_gpu_teacher import _check_distill, _check_top, _distill, _gen, _rows, _teacher, _top

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- attention

def test_recorded_attention_follows_its_inputs(mp):
    c = Case([200, 313, 0, 1], 4, 2, 64, window=150)
    ws = torch.empty(mp.mp_attention_bwd_workspace_bytes(c.T, 4, 2, 64), dtype=torch.uint8, device="cuda")
    run = lambda: (c.forward(mp), c.backward(mp, workspace=ws))  # noqa: E731
    run()
    grads = c.grads
    c.backward = lambda mp, **k: mp.mp_attention_bwd(c.do, c.q, c.k, c.v, c.o, c.lse, *grads, c.offsets, 4, 2, scale=c.scale, causal=True,
                                                     window=150, **k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    d = Case([200, 313, 0, 1], 4, 2, 64, window=150, seed=7)
    for name in ("q", "k", "v", "do"):
        getattr(c, name).copy_(getattr(d, name))
    c.offsets.copy_(torch.tensor([0, 50, 51, 400, 514], dtype=torch.int32))
    c.lengths = [50, 1, 349, 114]
    graph.replay()
    c.check_forward()
    Case.check_backward(c)


def test_two_streams_at_once_and_the_same_bits(mp):
    cs = [Case([700, 60], 8, 2, 128, seed=s) for s in range(2)]
    want = []
    for c in cs:
        c.forward(mp)
        c.backward(mp)
        want.append([t.clone() for t in (c.o, c.lse, *c.grads)])
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, c in zip(streams, cs):
            with torch.cuda.stream(s):
                c.forward(mp)
                c.backward(mp)
        torch.cuda.synchronize()
        for c, w in zip(cs, want):
            assert all(torch.equal(a, b) for a, b in zip((c.o, c.lse, *c.grads), w))


@pytest.mark.parametrize("D", [64, 128])
def test_thousands_of_tiny_sequences(mp, D):
    g = torch.Generator().manual_seed(0)
    c = Case(torch.randint(0, 4, (3000,), generator=g).tolist(), 1, 1, D, wide=True)
    c.forward(mp)
    c.backward(mp)
    # of one token: o = v, lse = its score, dv = do, dq = dk = 0
    at = torch.tensor([0] + c.lengths[:-1]).cumsum(0)
    one = at[torch.tensor(c.lengths) == 1].cuda()
    assert torch.equal(c.o[one], c.v[one])
    s = (c.q[one].double() * c.k[one].double()).sum(1) * c.scale
    assert bool(((c.lse[0, one].double() - s).abs() <= 2.0 ** -20 * (1 + s.abs())).all())
    small = H * c.do[one].abs().double().amax() + 2.0 ** -24
    assert bool(((c.grads[2][one].double() - c.do[one].double()).abs() <= small).all())
    # a row of one key: p = 1 to 2^-18, dp = delta to rounding, so ds is rounding alone
    assert c.grads[0][one].abs().max().item() <= 2.0 ** -8 and c.grads[1][one].abs().max().item() <= 2.0 ** -8


@pytest.mark.parametrize("causal", [True, False])
def test_values_of_other_sequences_never_matter(mp, causal):
    lengths = [130, 77, 300, 5]
    c = Case(lengths, 2, 1, 72, causal)
    c.forward(mp)
    c.backward(mp)
    clean = [t.clone() for t in (c.o, c.lse, *c.grads)]
    for t, bad in ((c.q, math.nan), (c.k, math.inf), (c.v, math.nan)):
        t[130:207] = bad                                     # the second sequence
    c.forward(mp)
    others = torch.ones(c.T, dtype=torch.bool, device="cuda")
    others[130:207] = False
    assert torch.equal(c.o[others], clean[0][others]) and torch.equal(c.lse[:, others], clean[1][:, others])
    assert bool(c.o[~others].isnan().all())
    # backward: its o and values are not finite, so ds is formed without the scale that fits them; the others stay right
    c.backward(mp)
    for got, want in zip(c.grads, clean[2:]):
        assert bool(got[others].isfinite().all())
        assert bool(((got[others].double() - want[others].double()).abs() <= 2.0 ** -8 * want[others].double().abs() + 2.0 ** -9).all())


@pytest.mark.parametrize("factor", [2.0 ** -14, 1.0, 2.0 ** 9])
def test_the_size_of_the_gradient_costs_no_bits(mp, factor):
    c = Case([400, 90], 2, 2, 64)
    c.do *= factor
    c.forward(mp)
    c.backward(mp)
    c.check_backward()


def test_attention_in_far_rows(mp):
    """Rows whose elements lie past 2^31 of the matrix."""
    T, pitch, n = 70_000, 32_768, 300
    full = torch.empty(T, pitch, dtype=torch.float16, device="cuda")
    c = Case([n], 1, 1, 64)
    mats = [full[:, 64 * i:64 * i + 64] for i in range(8)]
    q, k, v, do, o, dq, dk, dv = mats
    for t, src in ((q, c.q), (k, c.k), (v, c.v), (do, c.do)):
        t[T - n:] = src
    off = torch.tensor([T - n, T], dtype=torch.int64, device="cuda")
    lse = torch.empty(1, T, device="cuda")
    ws = torch.empty(mp.mp_attention_bwd_workspace_bytes(T, 1, 1, 64), dtype=torch.uint8, device="cuda")
    mp.mp_attention_fwd(q, k, v, o, lse, off, 1, 1)
    mp.mp_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, off, 1, 1, workspace=ws)
    c.forward(mp)
    c.backward(mp)
    assert torch.equal(o[T - n:], c.o) and torch.equal(lse[:, T - n:], c.lse)
    assert all(torch.equal(a[T - n:], b) for a, b in zip((dq, dk, dv), c.grads))


def test_attention_against_differences(mp):
    c = Case([40], 1, 1, 16, scale=0.25)
    c.forward(mp)
    c.backward(mp)
    h = 0.5
    vdo = (c.do.double() @ c.v.double().T).abs().max().item()

    def value():
        """sum do o, and what the rounding of the weights and of o may have done to it"""
        c.forward(mp)
        p = torch.softmax((c.q.double() @ c.k.double().T * 0.25).masked_fill(torch.ones(40, 40, device="cuda").triu(1).bool(), -math.inf), 1)
        return (c.do.double() * c.o.double()).sum().item(), (H * 1.02 * (c.do.double().abs() * (p @ c.v.double().abs() + c.o.double().abs())).sum()).item()
    for x, grad, other in ((c.q, c.grads[0], c.k), (c.k, c.grads[1], c.q)):
        for i, j in ((0, 0), (17, 5), (39, 15)):
            keep = x[i, j].item()
            x[i, j] = keep + h
            step = x[i, j].item() - keep
            up, e1 = value()
            x[i, j] = keep - h
            down, e2 = value()
            x[i, j] = keep
            diff = (up - down) / (2 * step)
            # a softmax's third derivatives are below 6 times the cube of what a step moves its scores by, for each row that it moves
            moved = (0.25 * other.double().abs()[:, j]) ** 3
            third = 6 * vdo * (moved.sum() if x is c.k else moved.max()).item()
            assert abs(diff - grad[i, j].item()) <= (e1 + e2) / (2 * step) + step * step / 6 * third + 2.0 ** -8


# ---------------------------------------------------------------- head norms

@pytest.mark.parametrize("k", [dict(T=40_000, hq=3, hk=1, D=32, rot=32), dict(T=9_001, hq=9, hk=4, D=128, rot=64, pairs=True),
                               dict(T=5_000, hq=20, hk=7, D=64, rot=64)], ids=lambda k: str(k["T"]))
def test_many_tokens_a_warp(mp, k):
    """Against calls of a few tokens: the same bits, and gradients of the gains over all tokens."""
    c = HeadCase(**k)
    y = torch.empty(c.x.shape, dtype=torch.float16, device="cuda")
    mp.mp_head_norm_rope_fwd(c.x, c.gq, c.gk, c.pos, c.freqs, y, c.hq, c.hk, pairs=c.pairs)
    ws = torch.empty(mp.mp_head_norm_rope_bwd_workspace_bytes(c.T, c.hq, c.hk, c.D), dtype=torch.uint8, device="cuda")
    dx, dg = torch.empty_like(y), [torch.empty(c.D, dtype=torch.float16, device="cuda") for _ in "qk"]
    mp.mp_head_norm_rope_bwd(c.dy, c.x, c.gq, c.gk, c.pos, c.freqs, dx, *dg, c.hq, c.hk, pairs=c.pairs, workspace=ws)
    few = [torch.empty_like(t) for t in dg]
    for a in list(range(0, c.T, max(c.T // 7, 1))) + [c.T - 3]:
        b = slice(a, a + 3)
        z = torch.empty_like(y[b])
        mp.mp_head_norm_rope_fwd(c.x[b], c.gq, c.gk, c.pos[b], c.freqs, z, c.hq, c.hk, pairs=c.pairs)
        assert torch.equal(z, y[b])
        mp.mp_head_norm_rope_bwd(c.dy[b], c.x[b], c.gq, c.gk, c.pos[b], c.freqs, z, *few, c.hq, c.hk, pairs=c.pairs, workspace=ws)
        assert torch.equal(z, dx[b])
    # Heads of one size in every element and gradients of 0, 1, -1: sums of multiples of r = 1 / sqrt(1 + eps), which FP32 does not
    # hold exactly, so that every addition may round.  A term passes through at most 400 additions (its lane's tokens and heads, at most
    # 60 here, the lanes, warps and blocks): 400 * 2^-24 of the sum of magnitudes, by the usual bound of a sum.
    c.x[:] = 1.0
    c.dy[:] = torch.randint(-1, 2, c.dy.shape, device="cuda").half()
    mp.mp_head_norm_rope_bwd(c.dy, c.x, c.gq, c.gk, None, None, dx, *dg, c.hq, c.hk, pairs=c.pairs, workspace=ws)
    u = c.dy.double().view(c.T, -1, c.D)
    for got, part in zip(dg, (u[:, :c.hq], u[:, c.hq:])):
        want = part.sum((0, 1))
        assert bool(((got.double() - want).abs() <= (H + 2.0 ** -19) * want.abs() + 400 * 2.0 ** -24 * part.abs().sum((0, 1))).all())


def test_head_norm_flags_and_streams(mp):
    c = HeadCase(T=100, hq=2, hk=1, D=64, rot=64)
    ws = torch.empty(mp.mp_head_norm_rope_bwd_workspace_bytes(100, 2, 1, 64), dtype=torch.uint8, device="cuda")
    dx, dg = torch.empty(c.x.shape, dtype=torch.float16, device="cuda"), [torch.empty(64, dtype=torch.float16, device="cuda") for _ in "qk"]
    st = mp.State(8.0)
    call = lambda: mp.mp_head_norm_rope_bwd(c.dy, c.x, c.gq, c.gk, c.pos, c.freqs, dx, *dg, 2, 1, state=st, workspace=ws)  # noqa: E731
    call()
    assert st.read().found_inf == 0
    want = [t.clone() for t in (dx, *dg)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in (dx, *dg):
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((dx, *dg), want))
    c.dy[50, 3] = math.inf
    call()
    assert st.read().found_inf == 1
    # no tokens: the gains' gradients are zeros
    mp.mp_head_norm_rope_bwd(c.dy[:0], c.x[:0], c.gq, c.gk, c.pos[:0], c.freqs, dx[:0], *dg, 2, 1, workspace=ws)
    assert not dg[0].any() and not dg[1].any()


# ---------------------------------------------------------------- scores and distillation

@pytest.mark.parametrize("N,V,k", [(9000, 29, 4), (2500, 700, 20), (3000, 1500, 128), (2500, 9000, 20), (1500, 20000, 64), (700, 50000, 128),
                                   (600, 140000, 20)])
def test_many_rows_a_worker(mp, N, V, k):
    g = _gen(N)
    z = _rows(g, N, V)
    w = (torch.rand(N, generator=g, device="cuda") < 0.8).float()
    w[:3] = 0
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    z[7::50] = 0.5                                           # rows of ties among the others
    _check_top(z, k, 1.0, _top(mp, z, k, 1.0, t, w), t, w)
    K = min(k, 31)
    ids, a = _teacher(g, z, K, 1.0)
    ids[5::40, 0] = -1
    got = _distill(mp, z, ids, a, w, 1.0, True, grad_scale=64.0)
    _check_distill(z, ids, a, w, 1.0, True, got, 64.0)


def test_concentrated_rows(mp):
    """All finite logits next to one another, the others -inf or FP16's lowest: one warp has every entry."""
    for V in (3000, 20000, 131071):
        for rest in (-math.inf, -65504.0):
            z = torch.full((6, -(-V // 8) * 8), rest, dtype=torch.float16, device="cuda")[:, :V]
            z[:, V // 2:V // 2 + 90] = torch.randn(6, 90, generator=_gen(V), device="cuda").half()
            for k in (20, 128):
                _check_top(z, k, 1.0, _top(mp, z, k))


def test_scores_and_losses_in_far_rows(mp):
    N, pitch, V = 40, 60_000_000, 3000
    full = torch.empty(N, pitch, dtype=torch.float16, device="cuda")
    z = full[:, :V]
    z[:] = torch.randn(N, V, generator=_gen(1), device="cuda").half()
    near = _rows(_gen(1), N, V)
    near[:] = z
    for a, b in zip(_top(mp, z, 9)[1:], _top(mp, near, 9)[1:]):
        assert torch.equal(a, b)
    ids, lp = _teacher(_gen(2), near, 9, 1.0)
    w = torch.ones(N, device="cuda")
    a, b = _distill(mp, z, ids, lp, w, out=full[:, 8000:8000 + V]), _distill(mp, near, ids, lp, w)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_recorded_scores_and_losses(mp):
    z = _rows(_gen(3), 200, 5000)
    ids, lp = torch.empty(200, 12, dtype=torch.int32, device="cuda"), torch.empty(200, 12, device="cuda")
    w, loss, total = torch.ones(200, device="cuda"), torch.empty(200, device="cuda"), torch.empty(1, device="cuda")
    dz = torch.empty(200, 5000, dtype=torch.float16, device="cuda")

    def run():
        mp.mp_token_top(z, ids, lp, temperature=2.0)
        mp.mp_distill_loss(z, ids, lp, w, loss, total, dz, 1.0, False, 16.0)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    z.copy_(_rows(_gen(4), 200, 5000))
    graph.replay()
    got = [t.clone() for t in (ids, lp, loss, total, dz)]
    run()
    assert all(torch.equal(a, b) for a, b in zip(got, (ids, lp, loss, total, dz)))
    _check_distill(z, ids, lp, w, 1.0, False, (dz, loss, total), 16.0)
