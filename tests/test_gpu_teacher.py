"""Token scores with top alternatives, and distillation from them, against the formulas in 64 bits.

Tolerances.  A log-probability is a difference of FP32 values as large as the largest |x| of its row (x = z / temperature), in
exponents of two: 2^-22 of it, and as much for the sum of V exponentials of two units in the last place.  An entropy is a
difference of such sums: 2^-19, and 2^-22 of it.  A stored FP16 gradient: half a step, 2^-11 of it (2^-25 below the normal range)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

H = 2.0 ** -11 * 1.001
S = 512.0


def _rows(g, N, V, std=2.0, extra=8):
    full = torch.full((N, -(-V // 8) * 8 + extra), float("nan"), dtype=torch.float16, device="cuda")
    full[:, :V] = torch.randn(N, V, generator=g, device="cuda") * std
    return full[:, :V]


def _gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---------------------------------------------------------------- scores

def _top(mp, z, k, temp=1.0, targets=None, weight=None, state=None):
    N = z.shape[0]
    out = [torch.full((N,), 7.0, device="cuda") for _ in range(2)]
    ids = torch.full((N, k), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((N, k), 7.0, device="cuda")
    mp.mp_token_top(z, ids, lp, targets=targets, logp=None if targets is None else out[0], entropy=out[1], weight=weight,
                    temperature=temp, state=state)
    return out[0], out[1], ids, lp


def _check_top(z, k, temp, got, targets=None, weight=None):
    logp, entropy, ids, lp = got
    for a in range(0, z.shape[0], 512):
        b = slice(a, a + 512)
        zz = z[b]
        on = torch.ones(len(zz), dtype=torch.bool, device="cuda") if weight is None else weight[b] != 0
        x = zz.double() / temp
        want = torch.log_softmax(x, 1)
        order = zz.float().sort(dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids[b], torch.where(on[:, None], order, -1).int())
        size = torch.where(x.isinf(), 0, x.abs()).amax(1)
        tol = 2.0 ** -20 + size * 2.0 ** -22 * 1.5
        w = want.gather(1, order)
        err = (lp[b].double() - torch.where(on[:, None], w, 0.0)).abs()
        err = torch.where(lp[b] == torch.where(on[:, None], w, 0.0), 0.0, err)          # -inf where it belongs
        assert bool((err <= tol[:, None]).all()), (err / tol[:, None]).max().item()
        h = -torch.where(want.isinf(), 0.0, want.exp() * want).sum(1)
        err = (entropy[b].double() - torch.where(on, h, 0.0)).abs()
        assert bool((err <= 2.0 ** -18 + tol).all()), (err / tol).max().item()
        if targets is not None:
            err = (logp[b].double() - torch.where(on, want.gather(1, targets[b][:, None].long())[:, 0], 0.0)).abs()
            assert bool((err <= tol).all()), (err / tol).max().item()


SIZES = [(1, 1, 1), (5, 2, 2), (9, 7, 3), (300, 29, 5), (33, 128, 128), (70, 256, 20), (20, 257, 1), (31, 600, 64), (17, 1024, 128),
         (13, 1025, 128), (13, 1032, 7), (200, 1500, 128), (9, 2047, 33), (150, 4097, 5), (170, 8192, 20), (160, 20001, 50),
         (3, 20001, 128), (5, 131071, 64), (150, 131071, 128), (2, 300000, 128), (1, 16385, 100)]


@pytest.mark.parametrize("N,V,k", SIZES)
def test_top(mp, N, V, k):
    g = _gen(V)
    z = _rows(g, N, V)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    temp = [1.0, 0.7, 2.0][V % 3]
    got = _top(mp, z, k, temp, t.int() if V % 2 else t)
    _check_top(z, k, temp, got, t)


# Rows shared by several blocks begin at these widths and end at these numbers of rows.
@pytest.mark.parametrize("N", [1, 74, 75, 148, 149])
@pytest.mark.parametrize("V", [4095, 4096, 8191, 8192, 16384, 16385, 32768, 32769, 65537])
def test_top_where_rows_are_shared(mp, N, V):
    z = _rows(_gen(N + V), N, V)
    for k in (1, 128):
        _check_top(z, k, 1.0, _top(mp, z, k))


@pytest.mark.parametrize("kind", ["equal", "steps", "rising", "falling", "minus_inf", "few", "zeros", "peak"])
@pytest.mark.parametrize("N,V,k", [(6, 29, 29), (6, 900, 100), (6, 5000, 128), (6, 40000, 64), (200, 40000, 64), (3, 131071, 128)])
def test_top_of_rows_that_defeat_a_bound(mp, kind, N, V, k):
    g = _gen(V + N)
    z = _rows(g, N, V)
    i = torch.arange(V, device="cuda")
    if kind == "equal":
        z[:] = 0.25
    elif kind == "steps":
        z[:] = (z * 2).round() / 2
    elif kind == "rising":
        z[:] = (i / V * 40 - 20).half()
    elif kind == "falling":
        z[:] = (20 - i / V * 40).half()
    elif kind == "minus_inf":
        z[:, V // 3:] = -math.inf
    elif kind == "few":                                      # fewer finite logits than k
        z[:] = -math.inf
        z[:, V // 2:V // 2 + 3] = 1.0
    elif kind == "zeros":                                    # two zeros are one value
        z[:] = torch.where(torch.rand(N, V, generator=g, device="cuda") < 0.5, 0.0, -0.0)
    else:
        z[:, V - 1] = 60000.0
    got = _top(mp, z, k)
    _check_top(z, k, 1.0, got)


def test_top_masked_rows_and_targets_out_of_range(mp):
    for V in (40, 3000, 20000):
        g = _gen(V)
        z = _rows(g, 50, V)
        weight = (torch.rand(50, generator=g, device="cuda") < 0.6).float()
        weight[3] = 1.0
        z[weight == 0] = math.nan                            # not read
        t = torch.randint(0, V, (50,), generator=g, device="cuda")
        t[weight == 0] = -5
        st = mp.State(S)
        got = _top(mp, z, 10, 1.0, t, weight, st)
        t0 = t.clamp(min=0)
        _check_top(torch.where(weight[:, None] == 0, 0.0, z), 10, 1.0, got, t0, weight)
        assert st.read().status == mp.MP_OK
        t[3] = V
        got = _top(mp, z, 10, 1.0, t, weight, st)
        assert math.isnan(got[0][3]) and not math.isnan(got[1][3]) and st.read().status == mp.MP_ERR_INVALID_ARG
        z[3, V // 2] = math.nan
        got = _top(mp, z, 10, 1.0, t0, weight)
        assert math.isnan(got[0][3]) and math.isnan(got[1][3]) and bool(got[3][3].isnan().all())
        assert bool(((got[2] >= -1) & (got[2] < V)).all())


def test_top_gives_the_same_bits(mp):
    z = _rows(_gen(), 300, 50000)
    a, b = _top(mp, z, 100), _top(mp, z, 100)
    assert all(torch.equal(x, y) for x, y in zip(a[1:], b[1:]))


# ---------------------------------------------------------------- distillation

def _teacher(g, z, K, temp):
    t = (z.float() + 0.7 * torch.randn(z.shape, generator=g, device="cuda")) / temp
    top = t.topk(K, 1)
    return top.indices, top.values - torch.logsumexp(t, 1, keepdim=True)


def _distill(mp, z, ids, a, w, temp=1.0, tail=True, state=None, grad_scale=S, out=None):
    N, V = z.shape
    loss, total = torch.full((N,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    dz = torch.full((N, -(-V // 8) * 8 + 8), 7.0, dtype=torch.float16, device="cuda")[:, :V] if out is None else out
    mp.mp_distill_loss(z, ids, a, w, loss, total, dz, temp, tail, grad_scale, state)
    return dz, loss, total


def _check_distill(z, ids, a, w, temp, tail, got, scale=S):
    dz, loss, total = got
    N, V = z.shape
    sum_tol = 0.0
    for s in range(0, N, 256):
        b = slice(s, s + 256)
        x = z[b].double() / temp
        lq = torch.log_softmax(x, 1)
        on = w[b] != 0
        has = ids[b] >= 0
        at = ids[b].long().clamp(min=0)
        listed = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
        rows = torch.arange(len(x), device="cuda")[:, None].expand_as(at)
        listed[rows[has], at[has]] = True
        aa = a[b].double().masked_fill(~has, -math.inf)
        if not tail:
            aa = aa - torch.logsumexp(aa, 1, keepdim=True)
            aa = torch.where(has.any(1, keepdim=True), aa, -math.inf)
        p = aa.exp()
        la = lq.gather(1, at)
        terms = torch.where(p > 0, p * (aa - la), 0.0)
        want, mag = terms.sum(1), torch.where(p > 0, p * (aa.abs() + la.abs()), 0.0).sum(1)
        mass, r, lr = p.sum(1), torch.zeros_like(want), torch.zeros_like(want)
        if tail:
            rest = lq.masked_fill(listed, -math.inf)
            lr = torch.logsumexp(rest, 1)
            r = torch.where(lr == -math.inf, 0.0, (1 - mass).clamp(min=0))
            t = torch.where(r > 0, r * (r.clamp(min=1e-300).log() - lr), 0.0)
            # r is a difference of FP32 sums: off by 2^-22, and its logarithm with it
            want, mag, mass = want + t, mag + t.abs() + (1 + (r.clamp(min=2.0 ** -23).log() - lr.clamp(min=-1e4)).abs()), mass + r
        q = lq.exp()
        grad = q * mass[:, None]
        soft = torch.where(lr[:, None] == -math.inf, 0.0, (lq - lr[:, None]).exp())          # of nothing: 0
        if tail:
            grad = torch.where(listed, grad, grad - torch.where(r[:, None] > 0, r[:, None] * soft, 0.0))
        hit = torch.zeros_like(q)
        hit[rows[has], at[has]] = p[has]
        G = scale / temp * w[b].double()[:, None]
        size = torch.where(x.isinf(), 0, x.abs()).amax(1, keepdim=True)
        rel = 2.0 ** -20 + size * 2.0 ** -22
        near = q * mass[:, None] + hit + (torch.where(listed, 0.0, (r[:, None] + 2.0 ** -22) * soft) if tail else 0.0)
        grad = torch.where(on[:, None], G * (grad - hit), 0.0)
        tol = G * near * rel * 3 + H * grad.abs() + 2.0 ** -25
        if tail:
            tol = tol + G * torch.where(listed, 0.0, soft) * 2.0 ** -21
        err = (dz[b].double() - grad).abs()
        err = torch.where(on[:, None], err, dz[b].double().abs())
        assert bool((err <= tol).all()), (err / tol).max().item()
        want = torch.where(on, w[b].double() * want, 0.0)
        ltol = torch.where(on, w[b].double() * (mag * 2.0 ** -20 + mass * (rel[:, 0] * 3)), 0.0)
        err = (loss[b].double() - want).abs()
        assert bool((err <= ltol + 1e-30).all()), (err / ltol).max().item()
        sum_tol += ltol.sum().item() + 2.0 ** -20 * want.abs().sum().item()
    assert abs(total.item() - loss.double().sum().item()) <= 2.0 ** -18 * loss.abs().double().sum().item() + 1e-30


DSIZES = [(1, 1, 1), (5, 2, 1), (7, 29, 29), (300, 29, 5), (40, 300, 64), (9, 2048, 128), (9, 2049, 20), (30, 5000, 33), (40, 20000, 20),
          (20, 33001, 128), (12, 70000, 64), (9, 131071, 128), (3, 300000, 7)]


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("N,V,K", DSIZES)
def test_distill(mp, N, V, K, tail):
    g = _gen(V + K)
    z = _rows(g, N, V)
    temp = [1.0, 0.7, 2.0][V % 3]
    ids, a = _teacher(g, z, K, temp)
    w = torch.where(torch.rand(N, generator=g, device="cuda") < 0.8, torch.rand(N, generator=g, device="cuda") + 0.1, 0.0)
    ids = ids.int() if V % 2 else ids
    z0 = z.clone()
    z[w == 0] = math.nan                                     # masked rows are not read
    got = _distill(mp, z, ids, a, w, temp, tail)
    _check_distill(z0, ids, a, w, temp, tail, got)
    full = got[0].as_strided((N, got[0].stride(0)), got[0].stride()) if N > 1 else got[0]
    assert bool((full[:, V:] == 7.0).all())
    # the gradient in the logits' place, and none: the same bits
    again = _distill(mp, z, ids, a, w, temp, tail, out=z)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


def test_distill_without_gradient_and_with_a_state(mp):
    g = _gen(5)
    z = _rows(g, 30, 5000)
    ids, a = _teacher(g, z, 10, 1.0)
    w = torch.full((30,), 1 / 30, device="cuda")
    st = mp.State(256.0)
    with_state = _distill(mp, z, ids, a, w, state=st, grad_scale=2.0)
    assert torch.equal(with_state[0], _distill(mp, z, ids, a, w, grad_scale=512.0)[0]) and st.read().found_inf == 0
    loss = torch.empty(30, device="cuda")
    mp.mp_distill_loss(z, ids, a, w, loss)
    assert torch.equal(loss, with_state[1])
    _distill(mp, z, ids, a, w, state=st, grad_scale=1e9)
    assert st.read().found_inf == 1


@pytest.mark.parametrize("V", [40, 3000, 40000, 131071])
@pytest.mark.parametrize("tail", [True, False])
def test_distill_lists_with_gaps(mp, V, tail):
    """Entries that are none, lists of nothing, probabilities of 0, a student that holds nearly everything in the list, rows whose
    other logits are -inf."""
    g = _gen(V)
    z = _rows(g, 12, V)
    ids, a = _teacher(g, z, 9, 1.0)
    ids[1, ::2] = -1
    ids[2] = -1
    a[3, 4] = -math.inf
    z[4, ids[4]] += 25.0                                     # the others: e^-20 of the row
    z[5] = -math.inf
    z[5, ids[5]] = 1.0
    a[6] += 3.0                                              # not normed: more than 1 in all
    z[7, :] = z[7] * 100
    w = torch.full((12,), 0.5, device="cuda")
    got = _distill(mp, z, ids, a, w, 1.0, tail, grad_scale=8.0)
    _check_distill(z, ids, a, w, 1.0, tail, got, 8.0)
    assert got[1][2].item() == 0.0 and bool((got[0][2] == 0).all())


@pytest.mark.parametrize("V", [40, 3000, 40000, 131071])
def test_distill_bad_lists(mp, V):
    g = _gen(V)
    z = _rows(g, 20, V)
    ids, a = _teacher(g, z, 9, 1.0)
    w = torch.ones(20, device="cuda")
    good = _distill(mp, z, ids, a, w)
    for row, col, value in ((3, 2, V), (5, 0, -2), (19, 8, None), (0, 1, None)):
        bad = ids.clone()
        bad[row, col] = bad[row, (col + 4) % 9] if value is None else value
        st = mp.State(1.0)
        dz, loss, total = _distill(mp, z, bad, a, w, state=st)
        assert bool(dz[row].isnan().all()) and math.isnan(loss[row]) and math.isnan(total)
        h = st.read()
        assert h.status == mp.MP_ERR_INVALID_ARG and h.found_inf == 1
        other = torch.arange(20, device="cuda") != row
        assert torch.equal(dz[other], good[0][other]) and torch.equal(loss[other], good[1][other])


def test_top_entries_of_the_teacher_feed_the_loss(mp):
    """A student that is its own teacher: no loss, and a gradient of rounding alone."""
    for V in (500, 20000):
        z = _rows(_gen(V), 64, V)
        for temp in (1.0, 2.0):
            _, _, ids, lp = _top(mp, z, 20, temp)
            w = torch.ones(64, device="cuda")
            dz, loss, _ = _distill(mp, z, ids, lp, w, temp, True, grad_scale=1.0)
            assert loss.abs().max().item() <= 2.0 ** -18 and dz.abs().max().item() <= 2.0 ** -18


def test_distill_gradient_against_differences(mp):
    g = _gen(9)
    V = 700
    z = (_rows(g, 1, V) * 4).round() / 4
    ids, a = _teacher(g, z, 12, 1.0)
    for tail in (True, False):
        one = torch.ones(1, device="cuda")
        dz = _distill(mp, z, ids, a, one, 1.0, tail, grad_scale=1.0)[0]
        for j in (int(ids[0, 0]), int(ids[0, 11]), int(z.argmin())):
            step = 0.125
            up, down = z.clone(), z.clone()
            up[0, j] += step
            down[0, j] -= step
            diff = (_distill(mp, up, ids, a, one, 1.0, tail)[1] - _distill(mp, down, ids, a, one, 1.0, tail)[1]).item() / (2 * step)
            # the third derivative of a log-sum is below 1: step^2 / 6 of it, and the FP32 losses' rounding
            assert abs(diff - dz[0, j].item()) <= step * step / 6 + 2.0 ** -17 / step
