"""The token-model kernels with many rows, blocks or tiles for each worker.

The kernels are persistent: a worker goes on to its next row or block while the copies of later ones are in flight.  The
sizes here give every worker several of them.  Three checks: the 64-bit formulas with the tolerances that
`test_gpu_token_ops` derives; the same bits as calls on so few rows that each worker has one; and inputs whose sums are
whole numbers below 2^24, so that FP32 holds them exactly and one row too many or too few shows.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_token_ops import (ADAMW, DEPTH, U, adamw64, close, gen, loss64, loss_inputs, norm64, norm_bwd64, norm_inputs,  # noqa: E402
                                out, padded, rand, up)


# ------------------------------------------------------------------------------ norms

# 148 blocks of 512 threads, 8 to 512 threads a row: 9472, 2368, 1184, 592, 296, 148 rows are one for each group
ROWS = [(40001, 64), (12011, 257), (6387, 1001), (3001, 1600), (1801, 2500), (901, 5000), (701, 9001)]
FORMS = [(0, 0, "shared"), (1, 1, "token"), (0, 1, "token"), (1, 0, "none"), (1, 0, "shared")]
FEW = 148                                                 # rows: one for each group at most


@pytest.mark.parametrize("M,D", ROWS)
@pytest.mark.parametrize("wide,kind,gate", FORMS)
def test_norm_forward_over_many_rows(mp, M, D, wide, kind, gate):
    eps, res = 1e-5, 0.75
    _, x, y, gp, gq, gt = norm_inputs(M, D, wide, gate, M + D)
    (xo, ok_x), (nn, ok_n), stats = out(M, D, x.dtype), out(M, D), torch.full((M, 4), 7.0, device="cuda")
    kw = dict(g_post16=gp, kind=kind, eps=eps, res_scale=res)
    mp.mp_block_norm_fwd(x, gq, nn, stats, y16=y, gate16=gt, x_out=xo, **kw)
    ok_x()
    ok_n()
    yhat, my, ry = norm64(y.double(), kind, eps)
    g64 = 1.0 if gt is None else gt.double()
    x64 = res * x.double() + yhat * gp.double() * g64
    xhat, mx, rx = norm64(x64, kind, eps)
    d = DEPTH * U
    size = lambda v, root: (v.abs() + v.abs().mean(1, keepdim=True)) * root  # noqa: E731  what cancels in v - mean
    err_x = d * (size(y.double(), ry) * gp.double() * g64).abs() + 4 * U * (res * x.double()).abs()
    close(xo, x64, err_x, "x_out")
    top = err_x.amax(1, keepdim=True)
    close(nn, xhat * gq.double(), (d * size(x64, rx) + 2 * top * rx * (1 + xhat.abs())) * gq.double().abs(), "n")
    few = lambda t, r: t[r:r + FEW] if t is not None and t.dim() == 2 else t  # noqa: E731
    xs, ns, ss = out(M, D, x.dtype)[0], out(M, D)[0], torch.empty(M, 4, device="cuda")
    for r in range(0, M, FEW):
        mp.mp_block_norm_fwd(few(x, r), gq, few(ns, r), few(ss, r), y16=few(y, r), gate16=few(gt, r), x_out=few(xs, r), **kw)
    assert torch.equal(xs, xo) and torch.equal(ns, nn) and torch.equal(ss, stats)
    x2, y2 = padded(x)[0], padded(y)[0]                   # in place
    mp.mp_block_norm_fwd(x2, gq, y2, None, y16=y2, gate16=gt, x_out=x2, **kw)
    assert torch.equal(x2, xo) and torch.equal(y2, nn)
    alone, s2 = out(M, D)[0], torch.empty(M, 4, device="cuda")          # the norm before the first block
    mp.mp_block_norm_fwd(x, gq, alone, s2, kind=kind, eps=eps)
    for r in range(0, M, FEW):
        mp.mp_block_norm_fwd(few(x, r), gq, few(ns, r), few(ss, r), kind=kind, eps=eps)
    assert torch.equal(alone, ns) and torch.equal(s2, ss)


@pytest.mark.parametrize("M,D", ROWS)
@pytest.mark.parametrize("wide,kind,gate", FORMS)
def test_norm_backward_over_many_rows(mp, M, D, wide, kind, gate):
    eps, res = 1e-5, 0.75
    g, xo, y, gp, gq, gt = norm_inputs(M, D, wide, gate, M + D + 1)
    dn = padded(rand(g, M, D, std=0.5))[0]
    above = padded(rand(g, M, D, std=0.5, dtype=xo.dtype))[0]
    stats = torch.cat(norm64(y.double(), kind, eps)[1:] + norm64(xo.double(), kind, eps)[1:], 1).float()
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda").fill_(0xFF)
    vec = lambda: out(1, D)[0][0]  # noqa: E731

    def call(rows, dn_, xo_, y_, gt_, up_, dx, dy, dgt):
        s = [vec() for _ in range(2)]
        mp.mp_block_norm_bwd(dn_, xo_, gq, stats[rows], dx, s[0], dx_out=up_, y16=y_, g_post16=gp, gate16=gt_, dy16=dy,
                             dg_post16=s[1], dgate16=dgt, kind=kind, res_scale=res, workspace=ws)
        return s
    new_gate = lambda: None if gt is None else vec() if gt.dim() == 1 else out(M, D)[0]  # noqa: E731
    every = slice(0, M)
    (dx, ok1), (dy, ok2), dgt = out(M, D, xo.dtype), out(M, D), new_gate()
    sums = call(every, dn, xo, y, gt, above, dx, dy, dgt)
    ok1()
    ok2()
    want = norm_bwd64(dn, xo, gq, stats.double(), above, y, gp, gt, kind, res)
    close(dx, *want["dx"], "dx")
    close(dy, *want["dy"], "dy")
    close(sums[0], *want["dg_pre"], "dg_pre")
    close(sums[1], *want["dg_post"], "dg_post")
    if gt is not None:
        close(dgt, *want["dgate"], "dgate")
    del want
    # the same bits in slices of a row a group (the sums over the rows have another order there)
    few = lambda t, r: t[r:r + FEW] if t is not None and t.dim() == 2 else t  # noqa: E731
    dxs, dys, dgs = out(M, D, xo.dtype)[0], out(M, D)[0], new_gate()
    for r in range(0, M, FEW):
        call(slice(r, r + FEW), few(dn, r), few(xo, r), few(y, r), few(gt, r), few(above, r), few(dxs, r), few(dys, r), few(dgs, r))
    assert torch.equal(dxs, dx) and torch.equal(dys, dy)
    matrix = gt is not None and gt.dim() == 2
    assert not matrix or torch.equal(dgs, dgt)
    # the same bits in the place of an input: dx at dx_out or x_out, dy at dn or y, a gate matrix's gradient at the gate
    for dx_at, dy_at, gate_at in (("up", "dn", False), ("xo", "y", True)):
        b = {"up": padded(above)[0], "xo": padded(xo)[0], "dn": padded(dn)[0], "y": padded(y)[0]}
        gt2 = padded(gt)[0] if matrix else gt
        dg2 = gt2 if matrix and gate_at else new_gate()
        again = call(every, b["dn"], b["xo"], b["y"], gt2, b["up"], b[dx_at], b[dy_at], dg2)
        assert torch.equal(b[dx_at], dx) and torch.equal(b[dy_at], dy) and (dgt is None or torch.equal(dg2, dgt))
        assert all(torch.equal(p, q) for p, q in zip(again, sums))


@pytest.mark.parametrize("M,D", ROWS)
@pytest.mark.parametrize("wide,gate", [(0, "shared"), (1, "token"), (1, "none")])
def test_norm_sums_over_the_rows_miss_none(mp, M, D, wide, gate):
    """Normed rows that are the stored ones (means 0, roots 1) and whole numbers throughout: the gradients of gains and gate
    are whole numbers that FP32 holds."""
    g = gen(M)
    whole = lambda hi, *s: torch.randint(-hi, hi + 1, s, generator=g, device="cuda")  # noqa: E731
    xt = torch.float32 if wide else torch.float16
    x, y, dn, above = whole(3, M, D), whole(3, M, D), whole(3, M, D), whole(3, M, D)
    gp, gq = torch.ones(D, dtype=torch.int64, device="cuda"), torch.ones(D, dtype=torch.int64, device="cuda")
    gt = None if gate == "none" else whole(2, D) if gate == "shared" else whole(2, M, D)
    stats = torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda").repeat(M, 1)
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    half = lambda t: None if t is None else padded(t.half())[0] if t.dim() == 2 else t.half()  # noqa: E731
    dx, dy = out(M, D, xt)[0], out(M, D)[0]
    dgp, dgq = (out(1, D)[0][0] for _ in range(2))
    dgt = None if gt is None else out(1, D)[0][0] if gt.dim() == 1 else out(M, D)[0]

    def call(dn_):
        mp.mp_block_norm_bwd(half(dn_), padded(x.to(xt))[0], half(gq), stats, dx, dgq, dx_out=padded(above.to(xt))[0], y16=half(y),
                             g_post16=half(gp), gate16=half(gt), dy16=dy, dg_post16=dgp, dgate16=dgt, workspace=ws)
    rounded = lambda t: t.double().half()  # noqa: E731
    call(dn)
    assert torch.equal(dgq, rounded((dn * x).sum(0)))
    call(torch.zeros_like(dn))                            # the gradient at x_out is then the one from above
    assert torch.equal(dx, above.to(xt))
    assert torch.equal(dgp, rounded((above * y * (1 if gt is None else gt)).sum(0)))
    if gt is not None:
        assert torch.equal(dgt, rounded((above * y).sum(0) if gt.dim() == 1 else above * y))


# ------------------------------------------------------------------------------ policy loss

# by the blocks of a row's cluster: 1, 1, 1, 2, 4, 8, 8; up to 1184 / blocks clusters work at once, and tokens are loaded for 32 rows
# of a cluster at a time
LOSS_ROWS = [(40009, 513), (9001, 5003), (5001, 16381), (14501, 20001), (7301, 40009), (3701, 70001), (1021, 131071)]


def masked(kind, N):
    i = torch.arange(N, device="cuda")
    return {"none": i < 0, "tenth": (i * 7919) % 10 == 0, "half": (i * 7919) % 2 == 0, "runs": (i // (N // 3 + 1)) % 2 == 1}[kind]


@pytest.mark.parametrize("N,V", LOSS_ROWS)
@pytest.mark.parametrize("kind", ["none", "tenth", "half", "runs"])
def test_policy_loss_over_many_rows(mp, N, V, kind):
    z, t, old, ref, adv, w = loss_inputs(8, V, V, True)
    g = gen(N)
    del z
    z = torch.empty(N, up(V) + 8, dtype=torch.float16, device="cuda")
    for r in range(0, N, 1024):
        z[r:r + 1024] = rand(g, min(1024, N - r), z.shape[1], std=2.0)
    z[:, V:] = float("nan")
    z = z[:, :V]
    pick = torch.arange(N, device="cuda") % 8
    t = (t[pick] + 31 * torch.arange(N, device="cuda")) % V
    lp0 = torch.cat([torch.log_softmax(z[r:r + 512].double(), 1).gather(1, t[r:r + 512, None])[:, 0] for r in range(0, N, 512)])
    ratio = torch.tensor([0.5, 0.79, 0.81, 0.9, 1.0, 1.1, 1.26, 1.3], device="cuda", dtype=torch.float64)[pick]
    old, ref = (lp0 - torch.log(ratio)).float(), (lp0 + 0.3 * torch.randn(N, generator=g, device="cuda")).float()
    adv, w = torch.randn(N, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda") + 0.5
    w[masked(kind, N)] = 0.0
    S = 256.0
    st = mp.State(init_scale=S)
    kw = dict(clip_lo=0.2, clip_hi=0.28, kl_coef=0.1, grad_scale=0.5, state=st)
    dz, ok = out(N, V)
    lp, tl, total = (torch.full((k,), 7.0, device="cuda") for k in (N, N, 1))
    mp.mp_policy_loss(z, t, old, adv, w, lp, tl, total, dlogits16=dz, ref_logp=ref, **kw)
    ok()
    if kind == "tenth":                                   # the others are compared with calls of few rows
        err = torch.zeros((), dtype=torch.float64, device="cuda")
        s = torch.zeros_like(err)
        for r in range(0, N, 512):
            k = slice(r, r + 512)
            want = loss64(z[k], t[k], old[k], ref[k], adv[k], w[k], 0.2, 0.28, 0.1, 0.5 * S, V)
            close(lp[k], *want["logp"], "logp")
            close(tl[k], *want["loss"], "loss")
            close(dz[k], *want["dz"], "dlogits")
            s += want["loss"][0].sum()
            err += want["loss"][1].sum() + DEPTH * U * want["loss"][0].abs().sum()
        close(total, s[None], err, "total")
    h = st.read()
    assert h.found_inf == 0 and h.status == 0
    few = 100                                             # clusters of a row each
    dzs, (lps, tls) = out(N, V)[0], (torch.empty(N, device="cuda") for _ in range(2))
    for r in range(0, N, few):
        k = slice(r, r + few)
        mp.mp_policy_loss(z[k], t[k], old[k], adv[k], w[k], lps[k], tls[k], dlogits16=dzs[k], ref_logp=ref[k], **kw)
    assert torch.equal(lps, lp) and torch.equal(tls, tl) and torch.equal(dzs, dz)
    del dzs
    lps.fill_(7.0)
    tls.fill_(7.0)
    mp.mp_policy_loss(z, t, old, adv, w, lps, tls, ref_logp=ref, **kw)                        # forward alone
    assert torch.equal(lps, lp) and torch.equal(tls, tl)
    lps.fill_(7.0)
    mp.mp_token_logp(z, t.int(), lps, weight=w)
    assert torch.equal(lps, lp)
    mp.mp_policy_loss(z, t, old, adv, w, lps, tls, dlogits16=z, ref_logp=ref, **kw)           # in the logits' place
    assert torch.equal(z, dz) and torch.equal(lps, lp) and torch.equal(tls, tl)
    st.close()


# ------------------------------------------------------------------------------ AdamW

def tensor_sizes(total):
    """Large tensors, 1500 small ones in a row, and odd sizes around the blocks of 256 and the units of 8 blocks."""
    g = torch.Generator().manual_seed(total)
    odd = [1, 255, 256, 257, 7 * 256 + 1, 8 * 256, 8 * 256 + 1, 15 * 256 - 1, 2047, 2049]
    small = torch.exp(torch.rand(1500, generator=g) * math.log(3000)).long().tolist()
    large = torch.exp(torch.rand(60, generator=g) * math.log(100))
    large = (large / large.sum() * (total - sum(small))).long().clamp(min=1).tolist()
    return large[:20] + odd + small[:900] + [0] + large[20:40] + small[900:] + large[40:] + odd[::-1]


class Flat:
    """Tensors as views of flat buffers with sevens between them, and the places of their elements and scales."""

    def __init__(self, counts, bits, seed):
        c = torch.tensor(counts)
        first = torch.cumsum((c + 15) // 16 * 16 + 16, 0) - ((c + 15) // 16 * 16 + 16) + 16
        blocks = (c + 255) // 256
        first_scale = torch.cumsum(blocks + 1, 0) - (blocks + 1) + 1
        of = torch.repeat_interleave(torch.arange(len(c)), c)
        pos = torch.arange(int(c.sum())) - torch.repeat_interleave(torch.cumsum(c, 0) - c, c)
        self.of, self.at, self.scale_at = of.cuda(), (first[of] + pos).cuda(), (first_scale[of] + pos // 256).cuda()
        size, scales = int(first[-1] + c[-1]) + 32, int(first_scale[-1] + blocks[-1]) + 1
        g = gen(seed)
        n = len(of)
        f8 = torch.float8_e4m3fn
        self.flat = {"g": rand(g, n, std=0.5), "w": rand(g, n, dtype=torch.float32)}
        self.flat["w16"] = self.flat["w"].half()
        if bits == 32:
            self.flat["m"], self.flat["v"] = 0.1 * rand(g, n, dtype=torch.float32), (0.05 * rand(g, n, dtype=torch.float32)) ** 2
        else:
            code = lambda: rand(g, n, std=60.0, dtype=torch.float32).clamp(-448, 448)  # noqa: E731
            self.flat["m"], self.flat["v"] = code().to(f8), code().abs().to(f8)
            for k in ("ms", "vs"):
                s = torch.full((scales,), 7.0, device="cuda")
                at = torch.unique(self.scale_at)
                s[at] = 1e-3 * (1 + torch.rand(len(at), generator=g, device="cuda"))
                self.flat[k] = s
        for k in ("g", "w", "w16", "m", "v"):
            full = torch.full((size,), 7.0, device="cuda").to(self.flat[k].dtype)
            full.view(torch.uint8 if full.dtype is f8 else full.dtype)[self.at] = \
                self.flat[k].view(torch.uint8 if full.dtype is f8 else full.dtype)
            self.flat[k] = full
        cut = lambda k: [self.flat[k][a:a + n] for a, n in zip(first.tolist(), counts)]  # noqa: E731
        cut_s = lambda k: [self.flat[k][a:a + n] for a, n in zip(first_scale.tolist(), blocks.tolist())] if bits == 8 else None  # noqa: E731
        self.views = [cut("g"), cut("w"), cut("m"), cut("v"), cut("w16"), cut_s("ms"), cut_s("vs")]

    def get(self, k):
        f = self.flat[k]
        return (f.view(torch.uint8)[self.at].view(f.dtype) if f.dtype is torch.float8_e4m3fn else f[self.at])

    def value(self, k, scale):
        v = self.get(k)
        return v.double() if scale not in self.flat else v.float().double() * self.flat[scale][self.scale_at].double()

    def untouched(self):
        for k in self.flat:
            f = self.flat[k].float()
            keep = torch.ones(len(f), dtype=torch.bool, device="cuda")
            keep[self.scale_at if k in ("ms", "vs") else self.at] = False
            assert (f[keep] == 7.0).all(), k

    def bytes(self):
        return {k: v.view(torch.uint8).clone() for k, v in self.flat.items()}


# 8 bits: units of 1, 2, 4 and 8 blocks of 256; 32 bits: always 1
@pytest.mark.parametrize("bits,total", [(8, 3_000_000), (8, 11_000_000), (8, 21_000_000), (8, 37_000_000), (32, 3_000_000), (32, 21_000_000)])
def test_adamw_over_many_blocks(mp, bits, total):
    counts = tensor_sizes(total)
    f = Flat(counts, bits, total % 1000)
    decay = [(0.0, 1.0, 0.5)[i % 3] for i in range(len(counts))]
    plan = mp.AdamWPlan(*f.views, decay)
    st = mp.State(init_scale=64.0, dynamic=False)
    opt = mp.AdamWConfig(**ADAMW)
    d = torch.tensor(decay, dtype=torch.float64, device="cuda")[f.of]
    for t in (1, 2):                                      # the second step reads the scales that the first one wrote
        w0, m0, v0 = f.get("w").clone(), f.value("m", "ms"), f.value("v", "vs")
        mp.mp_adamw_update(plan, st, opt, check_mode=t - 1)
        mp.mp_loss_scale_update(st)
        f.untouched()
        w, e_w, m, e_m, v, e_v = adamw64(f.get("g"), w0, m0, v0, t, 64.0, d, bits, **ADAMW)
        close(f.get("w"), w, e_w, "w")
        assert torch.equal(f.get("w16"), f.get("w").half())
        if bits == 32:
            close(f.get("m"), m, e_m, "m")
            close(f.get("v"), v, e_v, "v")
            continue
        r = torch.sqrt(v)
        for k, s, want, err, keep in (("m", "ms", m, e_m, False), ("v", "vs", r, 4 * U * r, True)):
            most = lambda x: torch.zeros(len(f.flat[s]), dtype=torch.float64, device="cuda").scatter_reduce(  # noqa: E731
                0, f.scale_at, x.abs(), "amax")
            live = torch.unique(f.scale_at)
            top, slack, scale = most(want)[live], most(err)[live], f.flat[s].double()[live]
            assert ((scale * 448 - top).abs() <= 8 * U * top + slack).all()
            step = f.flat[s].double()[f.scale_at]
            half = torch.maximum(want.abs() / 16, step * (2.0 ** -9 if keep else 2.0 ** -10))
            assert ((f.value(k, s) - want).abs() <= half * (1 + 1e-5) + err).all(), k
    assert st.read().t == 2
    # one infinity in the last element of a late tensor: found, and nothing is written
    late = f.views[0][len(counts) - 3]
    late[-1] = float("inf")
    before = f.bytes()
    mp.mp_adamw_update(plan, st, opt, check_mode=1)
    assert st.read().found_inf == 1 and all(torch.equal(a, before[k]) for k, a in f.bytes().items())
    plan.close()
    st.close()


# ------------------------------------------------------------------------------ embedding

@pytest.mark.parametrize("n,V,D", [(40000, 5000, 1024), (300007, 100, 72), (9001, 29, 4099)])
def test_embedding_of_a_large_batch(mp, n, V, D):
    g = gen(n)
    W = padded(rand(g, V, D))[0]
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    Y, untouched = out(n, D)
    mp.mp_embedding_fwd(ids, W, Y, pad_id=3, scale=3.5)
    want = (W.float() * 3.5).half()
    want[3] = 0
    assert torch.equal(Y, want[ids])
    untouched()


@pytest.mark.parametrize("n,V,D", [(25600, 29, 1600), (65537, 30000, 200), (200003, 400000, 24), (30000, 7, 4104), (1024, 60, 1000),
                                   (1025, 60, 1000), (16383, 5000, 264), (16384, 5000, 264)])
@pytest.mark.parametrize("kind", ["uniform", "zipf"])
def test_embedding_gradient_of_a_large_batch_misses_no_token(mp, n, V, D, kind):
    """Whole numbers: sums below 2^24 are exact in FP32, whatever the order."""
    g = gen(n + V)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = ((u * V).long() if kind == "uniform" else (torch.exp(u * math.log(V + 1)) - 1).long()).clamp_(0, V - 1)
    dY = padded(torch.randint(-3, 4, (n, D), generator=g, device="cuda").half())[0]
    want = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, ids, dY.double())
    dW, untouched = out(V, D)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda").fill_(0xFF)
    st = mp.State()
    mp.mp_embedding_bwd(ids, dY, dW, state=st, workspace=ws)
    assert torch.equal(dW, want.half())
    untouched()
    h = st.read()
    assert h.status == 0 and h.found_inf == 0
    st.close()
