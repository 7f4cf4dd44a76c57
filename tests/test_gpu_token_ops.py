"""The token-model operators against plain 64-bit statements of their formulas.

Tolerances.  u = 2^-24 is the unit roundoff of FP32, H = 2^-11 that of FP16 (and 2^-25 half its smallest
step).  A value that is stored once differs from its 64-bit value by the error of the FP32 arithmetic
before the store plus half a step of the stored type.  An FP32 sum of k terms is off by at most
depth * u * sum |terms|, depth <= k; the kernels add at most a few dozen terms in a row before they combine partial
sums, and DEPTH covers that and the handful of products around it.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, H, TINY = 2.0 ** -24, 2.0 ** -11, 2.0 ** -25
DEPTH = 200


def up(n, a=8):
    return -(-n // a) * a


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def padded(t, extra=8, fill=float("nan")):
    """The matrix t inside a wider buffer whose other columns hold `fill`; returns (view, buffer)."""
    r, c = t.shape
    buf = torch.full((r, up(c) + extra), fill, dtype=t.dtype, device="cuda")
    buf[:, :c] = t
    return buf[:, :c], buf


def out(r, c, dtype=torch.float16, extra=8):
    """An output view in a buffer of sevens, and a check that only the view was written."""
    buf = torch.full((r + 2, up(c) + extra), 7.0, dtype=dtype, device="cuda")
    view = buf[1:r + 1, :c]

    def untouched():
        assert (buf[0] == 7).all() and (buf[r + 1] == 7).all() and (buf[1:r + 1, c:] == 7).all()
    return view, untouched


def rand(g, *shape, std=1.0, mean=0.0, dtype=torch.float16):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


def close(got, want, err, what=""):
    """|got - want| within err (a tensor) plus half a step of got's type; infinities and NaN in the same places."""
    want = want.double()
    if got.dtype == torch.float16:                        # what FP16 cannot hold becomes an infinity
        want = torch.where(want.abs() >= 65520, torch.copysign(torch.full_like(want, math.inf), want), want)
    step = (H * want.abs() + TINY) if got.dtype == torch.float16 else U * want.abs()
    g = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), what
    assert torch.equal(g[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = (g - want).abs() - (err + step * (1 + 1e-9))
    off = off[fine]
    assert off.numel() == 0 or off.max().item() <= 0, (what, off.max().item(), int((off > 0).sum()))


# ------------------------------------------------------------------------------ embedding

IDS = [torch.int32, torch.int64]


@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 5, 8), (3, 7, 9), (16, 100, 1024), (37, 29, 1600), (5, 11, 4099),
                                   (2000, 3, 17), (0, 4, 8)])
def test_embedding_fwd(mp, n, V, D, wide):
    g = gen(n + V + D)
    W, _ = padded(rand(g, V, D))
    ids = torch.randint(0, V, (n,), generator=g, device="cuda").to(IDS[wide])
    pad = V // 2 if wide else -1
    Y, untouched = out(n, D)
    mp.mp_embedding_fwd(ids, W, Y, pad_id=pad, scale=math.sqrt(D))
    want = W.double()[ids.long()] * math.sqrt(D)
    want[ids == pad] = 0
    close(Y, want, 2 * U * want.abs())
    untouched()


def _embed_want(ids, dY, V, pad, scale):
    keep = (ids != pad).nonzero()[:, 0]
    acc = torch.zeros(V, dY.shape[1], dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(acc)
    acc.index_put_((ids.long()[keep],), dY.double()[keep], accumulate=True)
    mag.index_put_((ids.long()[keep],), dY.double()[keep].abs(), accumulate=True)
    return acc * scale, mag * abs(scale)


@pytest.mark.parametrize("kind", ["uniform", "zipf", "one", "padded"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 5, 8), (33, 7, 9), (300, 1000, 72), (700, 29, 1600), (5000, 700, 130),
                                   (2049, 2, 8), (20011, 40000, 24), (9000, 300000, 8), (70000, 520, 16), (0, 9, 16)])
def test_embedding_bwd(mp, n, V, D, kind):
    g = gen(n + V + D)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = (u * V).long() if kind in ("uniform", "padded") else (torch.exp(u * math.log(V + 1)) - 1).long()
    ids = ids.clamp_(0, V - 1)
    if kind == "one":
        ids = torch.full_like(ids, V - 1)
    pad = 0 if kind == "padded" else -1
    if kind == "padded":
        ids[n // 2:] = 0
    ids = ids.to(IDS[(n + V) % 2])
    dY, _ = padded(rand(g, n, D, std=0.1))
    dW, untouched = out(V, D)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda").fill_(0xFF)
    st = mp.State()
    want, mag = _embed_want(ids, dY, V, pad, 3.0)
    mp.mp_embedding_bwd(ids, dY, dW, pad_id=pad, scale=3.0, state=st, workspace=ws)
    close(dW, want, DEPTH * U * mag)
    untouched()
    h = st.read()
    assert h.status == 0 and h.found_inf == 0
    again = out(V, D)[0]                                  # any order of the work gives the same bits
    mp.mp_embedding_bwd(ids, dY, again, pad_id=pad, scale=3.0, workspace=ws)
    assert torch.equal(again, dW)
    st.close()


def test_embedding_bwd_is_the_gradient(mp):
    """sum(dY * lookup(W)) is linear in W: its differences are the gradient."""
    g = gen(3)
    n, V, D = 200, 31, 40
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    dY, W, Z = rand(g, n, D), rand(g, V, D), rand(g, V, D)
    dW, _ = out(V, D)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    mp.mp_embedding_bwd(ids, dY, dW, pad_id=4, scale=2.0, workspace=ws)
    F = lambda w: (dY.double() * w[ids] * 2.0 * (ids != 4)[:, None]).sum()  # noqa: E731
    h = 0.5
    diff = (F(W.double() + h * Z.double()) - F(W.double() - h * Z.double())) / (2 * h)
    _, mag = _embed_want(ids, dY, V, 4, 2.0)
    tol = ((H + DEPTH * U) * mag * Z.double().abs()).sum()
    assert abs((dW.double() * Z.double()).sum() - diff) <= tol


@pytest.mark.parametrize("wide", [0, 1])
def test_embedding_bad_ids(mp, wide):
    V, D = 10, 24
    W, dY = rand(gen(1), V, D), rand(gen(2), 6, D)
    ids = torch.tensor([3, -1, 10, 3, -5, 2 ** 31 - 1], device="cuda").to(IDS[wide])
    for pad in (-1, 3):
        st = mp.State()
        Y, untouched = out(6, D)
        mp.mp_embedding_fwd(ids, W, Y, pad_id=pad, state=st)
        untouched()
        assert st.read().status == mp.MP_ERR_INVALID_ARG
        assert torch.isnan(Y[[1, 2, 4, 5]]).all()
        assert torch.equal(Y[[0, 3]], W[[3, 3]] if pad < 0 else torch.zeros_like(W[[3, 3]]))
        st.close()
        st = mp.State()
        dW, untouched = out(V, D)
        ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(6, V, D), dtype=torch.uint8, device="cuda")
        mp.mp_embedding_bwd(ids, dY, dW, pad_id=pad, state=st, workspace=ws)
        untouched()
        assert st.read().status == mp.MP_ERR_INVALID_ARG
        want = torch.zeros(V, D, dtype=torch.float64, device="cuda")
        if pad < 0:
            want[3] = dY[0].double() + dY[3].double()
        close(dW, want, 4 * U * want.abs())
        st.close()
    # good ids leave the status alone, and a padding id outside the table is no error
    st = mp.State()
    Y, _ = out(2, D)
    mp.mp_embedding_fwd(torch.tensor([0, 50], device="cuda"), W, Y, pad_id=50, state=st)
    assert st.read().status == 0 and (Y[1] == 0).all()
    st.close()


def test_embedding_bwd_flags_overflow_and_ignores_the_padding_rows(mp):
    n, V, D = 64, 5, 16
    ids = torch.arange(n, device="cuda") % V
    dY = torch.ones(n, D, dtype=torch.float16, device="cuda")
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    for bad, pad, flag in ((float("nan"), -1, 1), (float("inf"), -1, 1), (60000.0, -1, 1), (float("nan"), 0, 0)):
        x = dY.clone()
        x[0, 3] = bad
        x[5, 3] = bad if bad == 60000.0 else 1.0
        st = mp.State()
        dW, _ = out(V, D)
        mp.mp_embedding_bwd(ids, x, dW, pad_id=pad, state=st, workspace=ws)
        assert st.read().found_inf == flag
        assert torch.isfinite(dW[1:]).all() and bool(torch.isfinite(dW[0]).all()) == (flag == 0)
        st.close()


def test_embedding_rows_past_32_bit_offsets(mp):
    V, D = 67000, 33000                                   # 2.2e9 elements
    W = torch.zeros(V, D, dtype=torch.float16, device="cuda")
    W[-1] = rand(gen(7), 1, D)[0]
    W[-2] = 2.0
    ids = torch.tensor([V - 1, V - 2, 0, V - 1], device="cuda")
    Y, _ = out(4, D)
    mp.mp_embedding_fwd(ids, W, Y)
    assert torch.equal(Y, W[ids])
    dY = rand(gen(8), 4, D)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(4, V, D), dtype=torch.uint8, device="cuda")
    W.fill_(7.0)
    mp.mp_embedding_bwd(ids, dY, W, workspace=ws)
    want = dY[0].double() + dY[3].double()
    close(W[-1], want, 4 * U * want.abs())
    assert torch.equal(W[-2], dY[1]) and torch.equal(W[0], dY[2])
    assert all(not W[a:min(a + 4096, V - 2)].any() for a in range(1, V - 2, 8192))


# ------------------------------------------------------------------------------ norms

def norm64(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind else torch.zeros_like(v[:, :1])
    root = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
    return (v - mean) * root, mean, root


NORM_SIZES = [(1, 1), (1, 8), (3, 5), (7, 33), (5, 256), (130, 257), (4, 1001), (19, 1024), (6, 2048), (3, 2500), (2, 4096),
              (3, 5000), (2, 8200), (2, 16384), (0, 16), (700, 64), (301, 1600)]


def norm_inputs(M, D, wide, gate, seed, offset=0.0):
    g = gen(seed)
    xt = torch.float32 if wide else torch.float16
    x, y = rand(g, M, D, std=3.0, mean=0.5 + offset, dtype=xt), rand(g, M, D, std=2.0, mean=-0.3)
    if M > 2:
        y[1], x[2] = 0.0, 0.0                             # rows without anything in them
    gains = [rand(g, D, std=0.2, mean=1.0) for _ in range(2)]
    gt = None if gate == "none" else rand(g, D, std=0.5) if gate == "shared" else padded(rand(g, M, D, std=0.5))[0]
    return g, padded(x)[0], padded(y)[0], gains[0], gains[1], gt


@pytest.mark.parametrize("M,D", NORM_SIZES)
@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("kind,gate", [(0, "shared"), (1, "token"), (0, "none")])
def test_block_norm_fwd(mp, M, D, wide, kind, gate):
    eps, res = 1e-5, 0.75
    _, x, y, gp, gq, gt = norm_inputs(M, D, wide, gate, M + D)
    xo, ok_x = out(M, D, x.dtype)
    nn, ok_n = out(M, D)
    stats = torch.full((M, 4), 7.0, device="cuda")
    mp.mp_block_norm_fwd(x, gq, nn, stats, y16=y, g_post16=gp, gate16=gt, x_out=xo, kind=kind, eps=eps, res_scale=res)
    yhat, my, ry = norm64(y.double(), kind, eps)
    g64 = 1.0 if gt is None else gt.double()
    h = yhat * gp.double() * g64
    x64 = res * x.double() + h
    xhat, mx, rx = norm64(x64, kind, eps)
    d = DEPTH * U
    size = lambda v, mean, root: (v.abs() + mean.abs()) * root  # noqa: E731  magnitude of what cancels in v - mean
    err_h = d * (size(y.double(), y.double().abs().mean(1, keepdim=True), ry) * gp.double() * g64).abs()
    err_x = err_h + 4 * U * (res * x.double()).abs()
    close(xo, x64, err_x, "x_out")
    top = err_x.amax(1, keepdim=True) if M else err_x[:, :1]
    spread = (d * size(x64, x64.abs().mean(1, keepdim=True), rx) + 2 * top * rx * (1 + xhat.abs())) * gq.double().abs()
    close(nn, xhat * gq.double(), spread, "n")
    mean_err = lambda v: d * v.abs().mean(1, keepdim=True)  # noqa: E731
    want = torch.cat([my, ry, mx, rx], 1)
    err = torch.cat([mean_err(y.double()), ry * d * 2 + ry * ry * mean_err(y.double()), mean_err(x64) + top,
                     rx * d * 2 + rx * rx * (mean_err(x64) + 2 * top)], 1)
    close(stats, want, err, "stats")
    ok_x()
    ok_n()
    # the same bits in place, on another stream, and without stats
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2, y2 = x.clone() if D % 8 == 0 else padded(x)[0], padded(y)[0]
        mp.mp_block_norm_fwd(x2, gq, y2, None, y16=y2, g_post16=gp, gate16=gt, x_out=x2, kind=kind, eps=eps, res_scale=res)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x2, xo) and torch.equal(y2, nn)


@pytest.mark.parametrize("M,D,wide,kind", [(1, 1, 0, 0), (5, 33, 0, 1), (3, 1024, 1, 0), (2, 16384, 0, 1), (9, 1600, 1, 1),
                                           (300, 64, 0, 0)])
def test_norm_before_the_first_block(mp, M, D, wide, kind):
    eps = 1e-6
    g, x, _, _, gq, _ = norm_inputs(M, D, wide, "none", 5)
    nn, ok = out(M, D)
    stats = torch.full((M, 4), 7.0, device="cuda")
    mp.mp_block_norm_fwd(x, gq, nn, stats, kind=kind, eps=eps)
    xhat, mx, rx = norm64(x.double(), kind, eps)
    size = (x.double().abs() + x.double().abs().mean(1, keepdim=True)) * rx
    close(nn, xhat * gq.double(), DEPTH * U * size * (1 + xhat.abs()) * gq.double().abs())
    ok()
    assert (stats[:, :2] == 0).all()
    dn = padded(rand(g, M, D))[0]
    st64 = torch.cat([torch.zeros(M, 2, device="cuda", dtype=torch.float64), mx, rx], 1)
    want = norm_bwd64(dn, x, gq, st64, None, None, None, None, kind, 1.0)
    dx, ok = out(M, D, x.dtype)
    dg = torch.empty(up(D), dtype=torch.float16, device="cuda")[:D]
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    mp.mp_block_norm_bwd(dn, x, gq, st64.float(), dx, dg, kind=kind, workspace=ws)
    close(dx, *want["dx"], "dx")
    close(dg, *want["dg_pre"], "dg_pre")
    ok()


def norm_bwd64(dn, xo, gq, stats, up_, y, gp, gt, kind, res):
    """Values and error bounds: each result with the magnitude of the terms that it is a sum of."""
    D = xo.shape[1]
    d = DEPTH * U
    mean = lambda v: v.sum(1, keepdim=True) / D  # noqa: E731

    def back(dv, err_dv, v, m, r):
        hat = (v - m) * r
        hat_mag = (v.abs() + m.abs()) * r
        p, q = mean(dv * hat), mean(dv) if kind else torch.zeros_like(m)
        val = (dv - hat * p - q) * r
        pm = mean(dv.abs() * hat_mag)
        mag = (dv.abs() + hat_mag * pm + mean(dv.abs())) * r
        e = (err_dv + hat_mag * mean(err_dv * hat_mag) + mean(err_dv)) * r
        return val, d * mag + e, hat, hat_mag

    dn, xo, gq = dn.double(), xo.double(), gq.double()
    zero = torch.zeros_like(dn)
    gx, e_gx, xhat, xmag = back(dn * gq, 2 * U * (dn * gq).abs(), xo, stats[:, 2:3], stats[:, 3:4])
    if up_ is not None:
        gx, e_gx = gx + up_.double(), e_gx + 4 * U * (up_.double().abs() + gx.abs())
    M = xo.shape[0]
    cols = lambda val, err: (val.sum(0), err.sum(0) + (DEPTH + M) * U * val.abs().sum(0))  # noqa: E731
    w = {"dg_pre": cols(dn * xhat, 8 * U * (dn.abs() * xmag))}
    if y is None:
        w["dx"] = (gx, e_gx)
        return w
    w["dx"] = (res * gx, abs(res) * e_gx + 2 * U * (res * gx).abs())
    y, gp = y.double(), gp.double()
    g64 = torch.ones_like(gp) if gt is None else gt.double()
    dh = gx * g64
    w["dy"] = back(dh * gp, (e_gx * g64 * gp).abs() + 4 * U * (dh * gp).abs(), y, stats[:, 0:1], stats[:, 1:2])[:2]
    yhat = (y - stats[:, 0:1]) * stats[:, 1:2]
    ymag = (y.abs() + stats[:, 0:1].abs()) * stats[:, 1:2]
    w["dg_post"] = cols(dh * yhat, (e_gx * g64).abs() * ymag + 8 * U * dh.abs() * ymag)
    one, e_one = gx * yhat * gp, (e_gx * ymag * gp.abs()) + 8 * U * (gx * gp).abs() * ymag
    if gt is not None:
        w["dgate"] = cols(one, e_one) if gt.dim() == 1 else (one, e_one + zero)
    return w


@pytest.mark.parametrize("M,D", NORM_SIZES)
@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("kind,gate,above", [(0, "shared", 1), (1, "token", 1), (0, "none", 0), (1, "shared", 0)])
def test_block_norm_bwd(mp, M, D, wide, kind, gate, above):
    eps, res = 1e-5, 0.75
    g, xo, y, gp, gq, gt = norm_inputs(M, D, wide, gate, M + D + 1)
    dn = padded(rand(g, M, D, std=0.5))[0]
    upg = padded(rand(g, M, D, std=0.5, dtype=xo.dtype))[0] if above else None
    st64 = torch.cat(norm64(y.double(), kind, eps)[1:] + norm64(xo.double(), kind, eps)[1:], 1)
    stats = st64.float()
    want = norm_bwd64(dn, xo, gq, stats.double(), upg, y, gp, gt, kind, res)
    vec = lambda: out(1, D)  # noqa: E731
    (dx, ok1), (dy, ok2), (dgp, ok3), (dgq, ok4) = out(M, D, xo.dtype), out(M, D), vec(), vec()
    dgt, ok5 = (None, lambda: None) if gt is None else vec() if gt.dim() == 1 else out(M, D)
    one = lambda t: t[0] if t is not None and gt is not None and gt.dim() == 1 else t  # noqa: E731
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda").fill_(0xFF)
    st = mp.State()

    def call(dx_, dy_, dgp_, dgq_, dgt_, up_, state=None):
        mp.mp_block_norm_bwd(dn, xo, gq, stats, dx_, dgq_, dx_out=up_, y16=y, g_post16=gp, gate16=gt, dy16=dy_,
                             dg_post16=dgp_, dgate16=dgt_, kind=kind, res_scale=res, state=state, workspace=ws)
    call(dx, dy, dgp[0], dgq[0], one(dgt), upg, st)
    close(dx, *want["dx"], "dx")
    close(dy, *want["dy"], "dy")
    close(dgq[0], *want["dg_pre"], "dg_pre")
    close(dgp[0], *want["dg_post"], "dg_post")
    if gt is not None:
        close(one(dgt), *want["dgate"], "dgate")
    for ok in (ok1, ok2, ok3, ok4, ok5):
        ok()
    assert st.read().found_inf == 0
    st.close()
    # the same bits where dx takes the place of dx_out
    if upg is not None:
        again = [torch.empty_like(t) for t in (dgp[0], dgq[0])]
        dy2 = out(M, D)[0]
        dgt2 = None if dgt is None else vec()[0][0] if gt.dim() == 1 else out(M, D)[0]
        call(upg, dy2, again[0], again[1], dgt2, upg)
        assert torch.equal(upg, dx) and torch.equal(dy2, dy) and torch.equal(again[0], dgp[0])
        assert torch.equal(again[1], dgq[0]) and (dgt is None or torch.equal(dgt2, one(dgt)))


@pytest.mark.parametrize("kind", [0, 1])
def test_block_norm_bwd_is_the_gradient(mp, kind):
    """Differences of the 64-bit forward pass along a random direction of every input."""
    M, D, eps, res = 6, 72, 1e-5, 0.75
    g, x, y, gp, gq, gt = norm_inputs(M, D, 1, "shared", 11)
    y[1], x[2] = 0.5 * y[0], 0.5 * x[0]
    xo = torch.empty_like(x)
    nn, stats = torch.empty(M, D, dtype=torch.float16, device="cuda"), torch.empty(M, 4, device="cuda")
    y = y.contiguous()
    mp.mp_block_norm_fwd(x, gq, nn, stats, y16=y, g_post16=gp, gate16=gt, x_out=xo, kind=kind, eps=eps, res_scale=res)
    dn, upg = rand(g, M, D), rand(g, M, D, dtype=torch.float32)

    def F(x, y, gp, gq, gt):
        o = res * x + gt * norm64(y, kind, eps)[0] * gp
        return (norm64(o, kind, eps)[0] * gq * dn.double()).sum() + (o * upg.double()).sum()
    at = [t.double() for t in (x, y, gp, gq, gt)]
    way = [torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for t in at]
    dx, dy = torch.empty(M, D, device="cuda"), torch.empty_like(nn)
    dgp, dgq, dgt = (torch.empty(D, dtype=torch.float16, device="cuda") for _ in range(3))
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    mp.mp_block_norm_bwd(dn, xo, gq, stats, dx, dgq, dx_out=upg, y16=y, g_post16=gp, gate16=gt, dy16=dy, dg_post16=dgp,
                         dgate16=dgt, kind=kind, res_scale=res, workspace=ws)
    for got, k in ((dx, 0), (dy, 1), (dgp, 2), (dgq, 3), (dgt, 4)):
        h = 1e-5
        move = lambda s: F(*[t + s * h * w if i == k else t for i, (t, w) in enumerate(zip(at, way))])  # noqa: E731
        diff = (move(1) - move(-1)) / (2 * h)
        # FP16 storage of the result, FP32 storage of x_out and stats, and h^2 of the difference
        tol = ((2 * H * got.double().abs() + 1e-4) * way[k].abs()).sum() + 1e-5
        assert abs((got.double() * way[k]).sum() - diff) <= tol, k


def test_block_norm_flags_and_nan_rows(mp):
    """A NaN in one row stays in that row; the gradients of the gains raise the flag."""
    M, D = 9, 264
    g, x, y, gp, gq, _ = norm_inputs(M, D, 0, "none", 2)
    y = y.contiguous()
    clean = [out(M, D)[0] for _ in range(2)]
    stats = torch.empty(M, 4, device="cuda")
    mp.mp_block_norm_fwd(x, gq, clean[1], stats, y16=y, g_post16=gp, x_out=clean[0])
    y[4, 100] = float("inf")
    dirty = [out(M, D)[0] for _ in range(2)]
    mp.mp_block_norm_fwd(x, gq, dirty[1], stats, y16=y, g_post16=gp, x_out=dirty[0])
    rest = [i for i in range(M) if i != 4]
    for a, b in zip(clean, dirty):
        assert torch.equal(a[rest], b[rest]) and torch.isnan(b[4]).any()
    st = mp.State()
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    dx, dy = out(M, D)[0], out(M, D)[0]
    dgp, dgq = (torch.empty(D, dtype=torch.float16, device="cuda") for _ in range(2))
    mp.mp_block_norm_bwd(rand(g, M, D), dirty[0], gq, stats, dx, dgq, y16=y, g_post16=gp, dy16=dy, dg_post16=dgp, state=st,
                         workspace=ws)
    assert st.read().found_inf == 1 and torch.isfinite(dx[rest]).all() and torch.isfinite(dy[rest]).all()
    st.close()


def test_block_norm_rows_past_32_bit_offsets(mp):
    M, D = 131100, 16384                                  # 2.15e9 elements
    x = torch.zeros(M, D, dtype=torch.float16, device="cuda")
    y = torch.zeros(M, D, dtype=torch.float16, device="cuda")
    g = gen(4)
    tail = rand(g, 3, D), rand(g, 3, D)
    x[-3:], y[-3:] = tail
    one = torch.ones(D, dtype=torch.float16, device="cuda")
    small = [torch.empty(3, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    s3, sM = torch.empty(3, 4, device="cuda"), torch.empty(M, 4, device="cuda")
    mp.mp_block_norm_fwd(tail[0], one, small[1], s3, y16=tail[1], g_post16=one, x_out=small[0])
    mp.mp_block_norm_fwd(x, one, y, sM, y16=y, g_post16=one, x_out=x)
    assert torch.equal(x[-3:], small[0]) and torch.equal(y[-3:], small[1]) and torch.equal(sM[-3:], s3)
    assert not x[0].any() and not y[70000].any()
    # backward over the same rows, in place: the gradient at x_out alone, then the whole block's
    dn = torch.zeros(M, D, dtype=torch.float16, device="cuda")
    dn[-3:] = rand(g, 3, D)
    y[-3:] = tail[1]
    ref = [torch.empty(3, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    dg = [torch.empty(D, dtype=torch.float16, device="cuda") for _ in range(4)]
    ws = torch.empty(max(mp.mp_block_norm_bwd_workspace_bytes(m, D) for m in (3, M)), dtype=torch.uint8, device="cuda")
    mp.mp_block_norm_bwd(dn[-3:].clone(), small[0], one, s3, ref[0], dg[0], dx_out=None, y16=tail[1], g_post16=one,
                         dy16=ref[1], dg_post16=dg[1], workspace=ws)
    mp.mp_block_norm_bwd(dn, x, one, sM, x, dg[2], dx_out=None, y16=y, g_post16=one, dy16=dn, dg_post16=dg[3], workspace=ws)
    assert torch.equal(x[-3:], ref[0]) and torch.equal(dn[-3:], ref[1])
    assert not x[0].any() and not dn[70000].any()


@pytest.mark.parametrize("M,D", [(1, 3), (9, 10), (40, 1001), (5, 2500), (3, 8201)])
@pytest.mark.parametrize("kind", [0, 1])
def test_fp32_rows_that_start_every_four_elements(mp, M, D, kind):
    """The FP32 residual with the narrowest pitch: the same bits as with a wide one, and nothing past the rows."""
    g, x, y, gp, gq, gt = norm_inputs(M, D, 1, "shared", 6)
    pitch = up(D, 4)

    def narrow(fill=None):
        buf = torch.full((M * pitch + 8,), 7.0, device="cuda")
        view = buf[:M * pitch].view(M, pitch)[:, :D]
        if fill is not None:
            view.copy_(fill)
        return view, lambda: bool((buf[M * pitch:] == 7).all() and (buf[:M * pitch].view(M, pitch)[:, D:] == 7).all())
    half = lambda: torch.zeros(M, up(D), dtype=torch.float16, device="cuda")[:, :D]  # noqa: E731
    vec = lambda: torch.zeros(up(D), dtype=torch.float16, device="cuda")[:D]  # noqa: E731
    y, dn, upg = y.contiguous() if D % 8 == 0 else padded(y)[0], padded(rand(g, M, D))[0], rand(g, M, D, dtype=torch.float32)
    ws = torch.empty(mp.mp_block_norm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    got = []
    for make in (narrow, lambda fill=None: (padded(fill)[0] if fill is not None else out(M, D, torch.float32)[0], lambda: True)):
        (xi, _), (xo, ok1), (ui, _), (dx, ok2) = make(x), make(), make(upg), make()
        nn, stats, dy = half(), torch.zeros(M, 4, device="cuda"), half()
        dg = [vec() for _ in range(3)]
        mp.mp_block_norm_fwd(xi, gq, nn, stats, y16=y, g_post16=gp, gate16=gt, x_out=xo, kind=kind)
        mp.mp_block_norm_bwd(dn, xo, gq, stats, dx, dg[0], dx_out=ui, y16=y, g_post16=gp, gate16=gt, dy16=dy, dg_post16=dg[1],
                             dgate16=dg[2], kind=kind, workspace=ws)
        assert ok1() and ok2()
        got.append([t.clone() for t in (xo, nn, stats, dx, dy, *dg)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ------------------------------------------------------------------------------ policy loss

def loss64(z, t, old, ref, adv, w, lo, hi, kl, scale, V):
    z = z.double()
    m = z.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))
    lp = z.gather(1, t[:, None])[:, 0] - lse[:, 0]
    r = torch.exp(lp - old.double())
    a, b = r * adv.double(), r.clamp(1 - lo, 1 + hi) * adv.double()
    loss, d = -torch.minimum(a, b), torch.where(a <= b, -a, 0.0)
    kd = torch.zeros_like(lp)
    if ref is not None:
        kd = ref.double() - lp
        loss, d = loss + kl * (torch.expm1(kd) - kd), d - kl * torch.expm1(kd)
    p = torch.exp(z - lse)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    c = scale * w.double() * d
    dz = c[:, None] * (hot - p)
    # errors: exp of an FP32 argument x is off by (2 |x| + 8) u relative; the sum by its depth besides
    e_lp = (V / 64 + 120) * U + 4 * U * (lp.abs() + (z.gather(1, t[:, None]) - m)[:, 0].abs())
    e_r = r * (e_lp + 4 * U * (lp - old.double()).abs() + 8 * U)
    e_k = kl * torch.exp(kd) * (e_lp + 4 * U * kd.abs() + 8 * U) + kl * 4 * U * kd.abs() if ref is not None else 0.0
    e_loss = w.double().abs() * (e_r * adv.double().abs() + 4 * U * loss.abs() + e_k)
    e_c = (scale * w.double()).abs() * (e_r * adv.double().abs() + e_k) + 4 * U * c.abs()
    e_dz = e_c[:, None] * (hot - p).abs() + c.abs()[:, None] * (
        torch.where(p > 0, p * ((2 * (z - lse).abs() + 16) * U + e_lp[:, None]), 0.0) + 2 * U * hot)
    live = w != 0
    zero = lambda v: torch.where(live if v.dim() == 1 else live[:, None], v, 0.0)  # noqa: E731
    return {"logp": (zero(lp), zero(e_lp)), "loss": (zero(w.double() * loss), zero(e_loss)), "dz": (zero(dz), zero(e_dz))}


def loss_inputs(N, V, seed, kl, std=2.0):
    g = gen(seed)
    z = rand(g, N, V, std=std)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, t[:, None])[:, 0]
    # ratios on both sides of the bounds 0.8 and 1.28 but never nearer to them than 1e-2
    pick = torch.tensor([0.5, 0.79, 0.81, 0.9, 1.0, 1.1, 1.26, 1.3, 2.0], device="cuda", dtype=torch.float64)
    ratio = pick[torch.randint(0, len(pick), (N,), generator=g, device="cuda")]
    old = (lp - torch.log(ratio)).float()
    ref = (lp + 0.3 * torch.randn(N, generator=g, device="cuda")).float() if kl else None
    adv = torch.randn(N, generator=g, device="cuda")
    w = torch.rand(N, generator=g, device="cuda") + 0.5
    w[torch.rand(N, generator=g, device="cuda") < 0.2] = 0.0
    return z, t, old, ref, adv, w


LOSS_SIZES = [(1, 1), (1, 2), (5, 7), (64, 29), (300, 64), (1000, 29), (33, 257), (7, 1000), (9, 4096), (5, 8193), (3, 32768),
              (4, 33001), (2, 65537), (3, 131071), (2, 200000), (1, 300000), (0, 16)]


@pytest.mark.parametrize("N,V", LOSS_SIZES)
@pytest.mark.parametrize("kl,wide", [(0.0, 1), (0.1, 0)])
def test_policy_loss(mp, N, V, kl, wide):
    z, t, old, ref, adv, w = loss_inputs(N, V, N + V, kl > 0)
    S = 256.0
    want = loss64(z, t, old, ref, adv, w, 0.2, 0.28, kl, 0.5 * S, V)
    zp = padded(z)[0]
    t = t.to(IDS[wide])
    dz, ok = out(N, V)
    lp, tl, total = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    st = mp.State(init_scale=S)
    kw = dict(ref_logp=ref, clip_lo=0.2, clip_hi=0.28, kl_coef=kl, grad_scale=0.5, state=st)
    mp.mp_policy_loss(zp, t, old, adv, w, lp, tl, total, dlogits16=dz, **kw)
    close(lp, *want["logp"], "logp")
    close(tl, *want["loss"], "loss")
    close(dz, *want["dz"], "dlogits")
    ok()
    s, e = want["loss"]
    close(total, s.sum()[None], e.sum() + (N + 8) * U * s.abs().sum(), "total")
    h = st.read()
    assert h.found_inf == 0 and h.status == 0
    # forward alone, the log-probabilities alone, and the gradient in the logits' place: the same bits
    lp2, tl2 = torch.empty_like(lp), torch.empty_like(tl)
    mp.mp_policy_loss(zp, t, old, adv, w, lp2, tl2, **kw)
    assert torch.equal(lp2, lp) and torch.equal(tl2, tl)
    mp.mp_token_logp(zp, t, lp2, weight=w)
    assert torch.equal(lp2, lp)
    mp.mp_policy_loss(zp, t, old, adv, w, lp2, tl2, dlogits16=zp, **kw)
    assert torch.equal(zp, dz) and torch.equal(lp2, lp)
    st.close()


@pytest.mark.parametrize("V", [29, 1000, 40000, 140000])
def test_policy_loss_hard_rows(mp, V):
    """Masked rows hold NaN and bad targets; live rows hold masked words (-inf and the lowest number), one
    word alone, huge logits, NaN, and targets out of range."""
    inf, nan = float("inf"), float("nan")
    N = 12
    z, t, old, ref, adv, w = loss_inputs(N, V, 1, True)
    w[:] = 1.0
    w[0] = w[5] = 0.0
    z[0], t[0], old[0] = nan, 2 ** 40, nan
    adv[5] = nan
    z[1, ::2], t[1] = -inf, 1
    z[2, ::2], t[2] = -65504.0, 1
    z[3], t[3] = -inf, V - 1
    z[3, V - 1] = 1.0
    z[4] = 60000.0 * torch.sign(z[4].float()).half()
    z[4, 0] = 60000.0
    t[4], old[4], ref[4] = 0, -1.0, -1.0
    for i in (1, 2, 3):
        lp = torch.log_softmax(z[i].double(), 0)[t[i]]
        old[i], ref[i] = lp, lp + 0.2
    z[6, V // 2] = nan
    t[7], t[8] = V, -1
    w[9] = nan
    z[10], t[10] = -inf, 0                                # every word masked: no distribution
    st = mp.State()
    dz, ok = out(N, V)
    lp, tl, total = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    mp.mp_policy_loss(padded(z)[0], t, old, adv, w, lp, tl, total, dlogits16=dz, ref_logp=ref, kl_coef=0.1, state=st)
    ok()
    h = st.read()
    assert h.status == mp.MP_ERR_INVALID_ARG and h.found_inf == 1
    st.close()
    good = [0, 1, 2, 3, 4, 5, 11]
    tt = t.clone()
    tt[[0, 7, 8]] = 0
    want = loss64(z, tt, old, ref, adv, w, 0.2, 0.2, 0.1, 65536.0, V)
    for name, got in (("logp", lp), ("loss", tl), ("dz", dz)):
        close(got[good], want[name][0][good], want[name][1][good], name)
    assert (dz[1, ::2] == 0).all() and (dz[0] == 0).all() and (dz[5] == 0).all()
    for i in (6, 7, 8, 10):
        assert torch.isnan(lp[i]) and torch.isnan(tl[i]) and torch.isnan(dz[i]).all(), i
    assert torch.isnan(tl[9]) and torch.isfinite(lp[9]) and torch.isnan(total).all()
    only = torch.empty(N, device="cuda")
    mp.mp_token_logp(padded(z)[0], t, only, weight=w)
    assert torch.equal(only.nan_to_num(5.0), lp.nan_to_num(5.0))
    # all rows masked
    mp.mp_policy_loss(padded(z)[0], t, old, adv, torch.zeros(N, device="cuda"), lp, tl, total, dlogits16=dz, ref_logp=ref)
    assert not dz.any() and not lp.any() and not tl.any() and total.item() == 0


def test_policy_loss_clip_edges(mp):
    """A = 0, and ratios exactly at 1 (where both branches agree): the gradient is that of r A."""
    V = 16
    z = torch.zeros(4, V, dtype=torch.float16, device="cuda")
    t = torch.arange(4, device="cuda")
    lp0 = torch.empty(4, device="cuda")
    mp.mp_token_logp(z, t, lp0)
    adv = torch.tensor([0.0, 1.0, -1.0, 2.0], device="cuda")
    lp, tl = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    dz = torch.empty_like(z)
    mp.mp_policy_loss(z, t, lp0, adv, torch.ones(4, device="cuda"), lp, tl, dlogits16=dz, clip_lo=0.0, clip_hi=0.0)
    assert torch.equal(tl, -adv)
    hot = torch.zeros(4, V, dtype=torch.float64, device="cuda").scatter_(1, t[:, None], 1.0)
    want = -adv.double()[:, None] * (hot - 1 / V)
    close(dz, want, 64 * U * want.abs())


def test_policy_loss_is_the_gradient(mp):
    N, V = 12, 300
    z, t, old, ref, adv, w = loss_inputs(N, V, 21, True)
    dz, lp, tl = torch.empty(N, up(V), dtype=torch.float16, device="cuda")[:, :V], *(torch.empty(N, device="cuda") for _ in "ab")
    mp.mp_policy_loss(padded(z)[0], t, old, adv, w, lp, tl, dlogits16=dz, ref_logp=ref, kl_coef=0.1, clip_hi=0.28)
    way = torch.randn(N, V, device="cuda", dtype=torch.float64, generator=gen(5))
    h = 1e-6
    F = lambda s: loss64(z.double() + s * h * way, t, old, ref, adv, w, 0.2, 0.28, 0.1, 1.0, V)["loss"][0].sum()  # noqa: E731
    diff = (F(1) - F(-1)) / (2 * h)
    tol = ((2 * H * dz.double().abs() + 2 * TINY) * way.abs()).sum() + 1e-6
    assert abs((dz.double() * way).sum() - diff) <= tol


def test_policy_loss_rows_past_32_bit_offsets(mp):
    N, V = 16400, 131072
    z = torch.zeros(N, V, dtype=torch.float16, device="cuda")
    tail, t3, old, ref, adv, w3 = loss_inputs(3, V, 9, True)
    w3[:] = 1.0
    z[-3:] = tail
    zero = torch.zeros(N - 3, device="cuda")
    cat = lambda a: torch.cat([zero, a])  # noqa: E731
    t = torch.cat([torch.zeros(N - 3, dtype=torch.int64, device="cuda"), t3])
    w = cat(w3)
    w[0] = 1.0
    lp, tl = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    mp.mp_policy_loss(z, t, cat(old), cat(adv), w, lp, tl, dlogits16=z, ref_logp=cat(ref), kl_coef=0.1)
    lp3, tl3, dz3 = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(tail)
    mp.mp_policy_loss(tail, t3, old, adv, w3, lp3, tl3, dlogits16=dz3, ref_logp=ref, kl_coef=0.1)
    assert torch.equal(z[-3:], dz3) and torch.equal(lp[-3:], lp3) and torch.equal(tl[-3:], tl3)
    assert not z[1:-3:1000].any() and abs(lp[0].item() + math.log(V)) < 1e-5


# ------------------------------------------------------------------------------ AdamW

def adamw_buffers(counts, seed, bits):
    g = gen(seed)
    b = {"g": [rand(g, c, std=0.5) for c in counts], "w": [rand(g, c, dtype=torch.float32) for c in counts]}
    b["w16"] = [w.half() for w in b["w"]]
    if bits == 32:
        b["m"] = [0.1 * rand(g, c, dtype=torch.float32) for c in counts]
        b["v"] = [(0.05 * rand(g, c, dtype=torch.float32)) ** 2 for c in counts]
        b["ms"] = b["vs"] = None
    else:
        b["m"] = [rand(g, c, std=60.0, dtype=torch.float32).clamp(-448, 448).to(torch.float8_e4m3fn) for c in counts]
        b["v"] = [rand(g, c, std=60.0, dtype=torch.float32).abs().clamp(max=448).to(torch.float8_e4m3fn) for c in counts]
        b["ms"] = [1e-3 * (1 + torch.rand(-(-c // 256), generator=g, device="cuda")) for c in counts]
        b["vs"] = [1e-3 * (1 + torch.rand(-(-c // 256), generator=g, device="cuda")) for c in counts]
    return b


def values(q, scale, c):
    return q.double() if scale is None else q.float().double() * scale.double().repeat_interleave(256)[:c]


ADAMW = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)


def adamw64(g, w, m, v_or_r, t, S, decay, bits, lr, beta1, beta2, eps, weight_decay):
    g = g.double() / S
    v = v_or_r if bits == 32 else v_or_r ** 2
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    w1 = w.double() * (1 - lr * weight_decay * decay)
    step = lr / (1 - beta1 ** t) * m1 / (torch.sqrt(v1 / (1 - beta2 ** t)) + eps)
    # m1 may cancel: its error is of the size of its terms
    e_m = 6 * U * (beta1 * m.abs() + (1 - beta1) * g.abs())
    e_w = 4 * U * w.double().abs() + 20 * U * step.abs() + \
        lr / (1 - beta1 ** t) * e_m / (torch.sqrt(v1 / (1 - beta2 ** t)) + eps)
    return w1 - step, e_w, m1, e_m, v1, 8 * U * v1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("counts", [[1], [7, 0, 8, 255, 256, 257], [1000, 3, 20000, 16], [2048 * 5], [8192 * 40 + 5, 1, 300]])
def test_adamw_steps(mp, counts, bits):
    b = adamw_buffers(counts, sum(counts), bits)
    decay = [1.0, 0.0, 0.5, 1.0, 0.0, 2.0][:len(counts)]
    plan = mp.AdamWPlan(b["g"], b["w"], b["m"], b["v"], b["w16"], b["ms"], b["vs"], decay)
    st = mp.State(init_scale=64.0, dynamic=False)
    opt = mp.AdamWConfig(**ADAMW)
    for t in (1, 2, 3):
        old = [(b["w"][i].clone(), values(b["m"][i], b["ms"] and b["ms"][i], c), values(b["v"][i], b["vs"] and b["vs"][i], c))
               for i, c in enumerate(counts)]
        mp.mp_adamw_update(plan, st, opt)
        mp.mp_loss_scale_update(st)
        for i, c in enumerate(counts):
            if c == 0:
                continue
            w0, m0, v0 = old[i]
            w, e_w, m, e_m, v, e_v = adamw64(b["g"][i], w0, m0, v0, t, 64.0, decay[i], bits, **ADAMW)
            close(b["w"][i], w, e_w, "w")
            assert torch.equal(b["w16"][i], b["w"][i].half())
            if bits == 32:
                close(b["m"][i], m, e_m, "m")
                close(b["v"][i], v, e_v, "v")
                continue
            pad = lambda x: torch.nn.functional.pad(x, (0, -c % 256)).view(-1, 256)  # noqa: E731
            r = torch.sqrt(v)
            for q, scale, want, err, keep in ((b["m"][i], b["ms"][i], m, e_m, False), (b["v"][i], b["vs"][i], r, 4 * U * r, True)):
                top = pad(want).abs().amax(1)
                assert ((scale.double() * 448 - top).abs() <= 8 * U * top + pad(err).amax(1)).all()
                step = scale.double().repeat_interleave(256)[:c]
                # half a step of E4M3: 2^-4 relative above 2^-6, 2^-10 below (a kept r: up to 2^-9)
                half = torch.maximum(want.abs() / 16, step * (2.0 ** -9 if keep else 2.0 ** -10))
                off = (values(q, scale, c) - want).abs()
                assert (off <= half * (1 + 1e-5) + err).all()
                if keep:
                    assert ((q.float() > 0) == (want > 0)).all()
    assert st.read().t == 3
    plan.close()
    st.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_overflow_step_writes_nothing(mp, bits):
    counts = [300, 5000]
    b = adamw_buffers(counts, 1, bits)
    b["g"][1][4999] = float("inf")
    plan = mp.AdamWPlan(b["g"], b["w"], b["m"], b["v"], b["w16"], b["ms"], b["vs"])
    raw = lambda t: t.view(torch.uint8).clone()  # noqa: E731
    keep = [raw(t) for k in ("w", "m", "v", "w16", "ms", "vs") if b[k] for t in b[k]]
    now = lambda: [raw(t) for k in ("w", "m", "v", "w16", "ms", "vs") if b[k] for t in b[k]]  # noqa: E731
    st = mp.State(init_scale=64.0)
    mp.mp_adamw_update(plan, st, mp.AdamWConfig(**ADAMW), check_mode=1)      # finds the inf itself
    assert st.read().found_inf == 1
    mp.mp_loss_scale_update(st)
    h = st.read()
    assert (h.scale, h.t, h.skipped) == (32.0, 0, 1)
    assert all(torch.equal(a, c) for a, c in zip(keep, now()))
    # a device-side error freezes it as well
    h.status = mp.MP_ERR_INVALID_ARG
    st.write(h)
    b["g"][1][4999] = 1.0
    mp.mp_adamw_update(plan, st, mp.AdamWConfig(**ADAMW), check_mode=1)
    assert all(torch.equal(a, c) for a, c in zip(keep, now()))
    h.status = 0
    st.write(h)
    mp.mp_adamw_update(plan, st, mp.AdamWConfig(**ADAMW), check_mode=1)
    assert not any(torch.equal(a, c) for a, c in zip(keep[:2], now()[:2]))
    plan.close()
    st.close()


def test_adamw_8bit_from_zero_and_idle_blocks(mp):
    """All-zero states are the start; a block without gradients stays zero and its weights only decay."""
    c = 256 * 6 + 40
    g = torch.zeros(c, dtype=torch.float16, device="cuda")
    g[256:512] = rand(gen(1), 256)
    g[600] = 1e-7                                         # a lone, tiny gradient in its block
    g[1536:] = 6e4
    w = rand(gen(2), c, dtype=torch.float32)
    w0 = w.clone()
    m, v = (torch.zeros(c, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ms, vs = torch.zeros(7, device="cuda"), torch.zeros(7, device="cuda")
    w16 = torch.empty_like(g)
    plan = mp.AdamWPlan([g], [w], [m], [v], [w16], [ms], [vs])
    st = mp.State(init_scale=1.0, dynamic=False)
    mp.mp_adamw_update(plan, st, mp.AdamWConfig(**ADAMW))
    idle = torch.tensor([0, 3, 4, 5], device="cuda")
    assert not ms[idle].any() and not vs[idle].any() and (ms[[1, 2, 6]] > 0).all() and (vs[[1, 2, 6]] > 0).all()
    want, e_w, *_ = adamw64(g, w0, torch.zeros(c, dtype=torch.float64, device="cuda"),
                            torch.zeros(c, dtype=torch.float64, device="cuda"), 1, 1.0, 1.0, 8, **ADAMW)
    close(w, want, e_w)
    assert m.float()[600] == 448 and v.float()[600] == 448
    plan.close()
    st.close()


def test_adamw_long_run_8bit_follows_32bit(mp):
    """A quadratic bowl: the 8-bit states reach the minimum about as closely as the 32-bit ones."""
    c = 4096
    target = rand(gen(1), c, dtype=torch.float32)
    far = {}
    for bits in (32, 8):
        w = torch.zeros(c, device="cuda")
        w16, g = w.half(), torch.empty(c, dtype=torch.float16, device="cuda")
        st = torch.float32 if bits == 32 else torch.float8_e4m3fn
        m, v = torch.zeros(c, dtype=torch.float32, device="cuda").to(st), torch.zeros(c, device="cuda").to(st)
        ms = vs = None
        if bits == 8:
            ms, vs = [torch.zeros(16, device="cuda")], [torch.zeros(16, device="cuda")]
        plan = mp.AdamWPlan([g], [w], [m], [v], [w16], ms, vs)
        state = mp.State(init_scale=8.0, dynamic=False)
        for i in range(1000):                             # the learning rates sum to 10, every target lies within 4
            opt = mp.AdamWConfig(lr=0.02 * (1 - i / 1000), beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
            g.copy_((w - target) * 8.0)
            mp.mp_adamw_update(plan, state, opt)
            mp.mp_loss_scale_update(state)
        far[bits] = (w - target).abs().max().item()
        plan.close()
        state.close()
    assert far[32] < 0.05 and far[8] < 0.05, far


def test_binding_refuses_wrong_types_and_shapes(mp):
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        mp.mp_embedding_fwd(ids.float(), h(5, 8), h(4, 8))
    with pytest.raises(ValueError):
        mp.mp_embedding_fwd(ids, h(5, 8), h(3, 8))
    with pytest.raises(TypeError):
        mp.mp_embedding_bwd(ids, f(4, 8), h(5, 8))
    with pytest.raises(mp.MpError):
        mp.mp_embedding_bwd(ids, h(4, 8), h(5, 8))                          # no workspace
    with pytest.raises(mp.MpError):
        mp.mp_embedding_fwd(ids, h(5, 9), h(4, 9))                          # pitch 9
    with pytest.raises(TypeError):
        mp.mp_block_norm_fwd(f(4, 8), h(8), h(4, 8), y16=h(4, 8), g_post16=h(8), x_out=h(4, 8))
    with pytest.raises(ValueError):
        mp.mp_block_norm_fwd(h(4, 8), h(9), h(4, 8))
    with pytest.raises(ValueError):
        mp.mp_policy_loss(h(4, 8), ids[:3], f(4), f(4), f(4), f(4), f(4))
    with pytest.raises(ValueError):
        mp.mp_policy_loss(h(4, 8), ids, f(3), f(4), f(4), f(4), f(4))
    with pytest.raises(ValueError):
        mp.AdamWPlan([h(8)], [f(9)], [f(8)], [f(8)], [h(8)])
    with pytest.raises(TypeError):
        mp.AdamWPlan([h(8)], [f(8)], [f(8)], [f(8)], [h(8)], m_scale=[f(1)], v_scale=[f(1)])
