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


def test_calls_that_follow_one_another_in_one_workspace(mp):
    """Batches whose long runs lie elsewhere, one after the other without a pause: no call may see the sorted
    tokens or the partial rows of the call before it."""
    V, D, n = 900, 200, 30000
    g = torch.Generator(device="cuda").manual_seed(3)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    cases = []
    for k in range(8):                                    # exact sums: small whole numbers
        ids = torch.randint(0, V, (n,), generator=g, device="cuda")
        start = 3000 * k
        ids[start:start + 9000] = (131 * k) % V
        dY = torch.randint(-2, 3, (n, D), generator=g, device="cuda").half()
        want = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, ids, dY.double())
        cases.append((ids, dY, want.half()))
    outs = [torch.full((V, D), 7.0, dtype=torch.float16, device="cuda") for _ in range(80)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        mp.mp_embedding_bwd(cases[i % 8][0], cases[i % 8][1], o, workspace=ws)
    assert all(torch.equal(o, cases[i % 8][2]) for i, o in enumerate(outs))


def test_embedding_gradient_of_rows_wider_than_a_grid_is_high(mp):
    """17 million columns: more blocks over the columns than a grid's second dimension holds.  Whole numbers, so exact."""
    n, V, D = 300, 2, 17_000_008
    dY = torch.empty(n, D, dtype=torch.float16, device="cuda")
    col = torch.arange(D, device="cuda", dtype=torch.int32)
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    ids[::3] = 1                                          # runs of 100 and 200 tokens: over one tile, over three
    ids = 1 - ids
    want = torch.zeros(V, D, dtype=torch.float32, device="cuda")
    rows = ids.tolist()
    for i in range(n):
        dY[i] = ((col + 7 * i) % 5 - 2).half()
        want[rows[i]] += dY[i].float()
    dW = torch.full((V, D), 7.0, dtype=torch.float16, device="cuda")
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    mp.mp_embedding_bwd(ids, dY, dW, workspace=ws)
    assert torch.equal(dW, want.half())


@pytest.mark.parametrize("M,D,wide", [(5, 1, 0), (9, 33, 1), (3, 1001, 0), (2, 2501, 1), (2, 9001, 0)])
@pytest.mark.parametrize("kind", [0, 1])
def test_what_follows_gains_and_gates_does_not_matter(mp, M, D, wide, kind):
    """Vectors whose length is no multiple of 8, with NaN behind them and with zeros: the same bits, and none of it written."""
    g = torch.Generator(device="cuda").manual_seed(D)
    wide_d = -(-D // 8) * 8
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").half()  # noqa: E731
    mats = {k: rnd(M, wide_d)[:, :D] for k in ("y", "dn")}
    xt = torch.float32 if wide else torch.float16
    x, up = (torch.randn(M, wide_d, generator=g, device="cuda").to(xt)[:, :D] for _ in range(2))
    vecs = [rnd(D) for _ in range(3)]
    results = []
    for fill in (float("nan"), 0.0):
        def vec(v=None):
            b = torch.full((wide_d + 8,), fill, dtype=torch.float16, device="cuda")
            if v is not None:
                b[:D] = v
            return b
        bufs = [vec(v) for v in vecs]
        gp, gq, gt = (b[:D] for b in bufs)
        outs = [vec() for _ in range(3)]
        new = lambda t: torch.zeros(M, wide_d, dtype=t, device="cuda")[:, :D]  # noqa: E731
        xo, n, dx, dy, stats = new(xt), new(torch.float16), new(xt), new(torch.float16), torch.zeros(M, 4, device="cuda")
        ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
        mp.mp_block_norm_fwd(x, gq, n, stats, y16=mats["y"], g_post16=gp, gate16=gt, x_out=xo, kind=kind)
        mp.mp_block_norm_bwd(mats["dn"], xo, gq, stats, dx, outs[0][:D], dx_out=up, y16=mats["y"], g_post16=gp, gate16=gt, dy16=dy,
                             dg_post16=outs[1][:D], dgate16=outs[2][:D], kind=kind, workspace=ws)
        for b in bufs + outs:
            assert torch.isnan(b[D:]).all() if fill != fill else not b[D:].any()
        results.append([t.clone() for t in (xo, n, dx, dy, stats, *(o[:D] for o in outs))])
    assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(*results))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_of_masked_tokens_alone_decays_the_matrices(mp, bits):
    """No gradient and first moments of zero: the matrices shrink by 1 - lr weight_decay, gains and gates keep their bits."""
    from paper_1805_10387_b200.token_model import TokenModel
    n, V, lr, decay = 64, 50, 1e-2, 0.25
    model = TokenModel(V, 64, 64, 1, n, init_scale=1024.0, state_bits=bits, lr=lr, weight_decay=decay)
    ids = torch.arange(n, device="cuda") % V
    one, lp = torch.ones(n, device="cuda"), torch.empty(n, device="cuda")
    model.log_probs(ids, ids, lp)
    for _ in range(2):
        model.step(ids, ids, lp, one, one / n)
    for t in model.flat["m"] + model.flat["ms"]:
        t.view(torch.uint8).zero_()
    before = {k: v.clone() for k, v in model.w32.items()}
    model.step(ids, ids, lp, one, 0 * one)
    h = model.state.read()
    assert h.t == 3 and h.skipped == 0 and model.loss.item() == 0
    for k, w in model.w32.items():
        assert not model.dw[k].any(), k
        if w.dim() == 1:
            assert torch.equal(w, before[k]), k
        else:                                             # the factor, its product and the difference are rounded
            want = before[k].double() * (1 - lr * decay)
            assert ((w.double() - want).abs() <= U * want.abs() + 2 * U * lr * decay * before[k].double().abs() + 1e-45).all(), k
            assert not torch.equal(w, before[k])
    model.close()


@pytest.mark.parametrize("n,V", [(700, 2 ** 21 - 1), (700, 2 ** 21), (1024, 20_000_000), (5, 2 ** 24 + 1), (3000, 2 ** 24)])
def test_embedding_gradient_of_few_tokens_in_a_huge_table(mp, n, V):
    """Id and position of a token fit one word up to 2^21 rows; from there on, and past 2^24, the sort takes three and four passes."""
    D = 8
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    ids[:2], ids[n // 2:n // 2 + 2], ids[-1] = V - 1, 0, V - 1
    dY = torch.randint(-3, 4, (n, D), generator=g, device="cuda").half()
    want = torch.zeros(V, D, dtype=torch.float16, device="cuda")
    some, where = torch.unique(ids, return_inverse=True)
    want[some] = torch.zeros(len(some), D, dtype=torch.float64, device="cuda").index_add_(0, where, dY.double()).half()
    dW = torch.full((V, D), 7.0, dtype=torch.float16, device="cuda")
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda").fill_(0xFF)
    mp.mp_embedding_bwd(ids, dY, dW, workspace=ws)
    assert torch.equal(dW, want)
