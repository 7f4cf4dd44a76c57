"""Refusals of the token-model calls: every bad argument is found on the host, before any CUDA call."""
import ctypes as C

import pytest

from paper_1805_10387_b200 import mp


_BUF = (C.c_uint16 * 4096)()


@pytest.fixture
def p16():
    """A 16-byte aligned host address: no call of this file gets as far as reading it."""
    return (C.addressof(_BUF) + 15) // 16 * 16


def _embed_fwd(L, p, **k):
    a = dict(ids=p, idb=8, W=p, ldw=8, Y=p, ldy=8, n=4, V=4, D=8)
    a.update(k)
    return L.mp_embedding_fwd(a["ids"], a["idb"], a["W"], a["ldw"], a["Y"], a["ldy"], a["n"], a["V"], a["D"], -1, 1.0,
                              None, None)


def _embed_bwd(L, p, **k):
    a = dict(ids=p, idb=8, dY=p, lddy=8, dW=p, ldw=8, n=4, V=4, D=8, ws=p, nb=1 << 40)
    a.update(k)
    return L.mp_embedding_bwd(a["ids"], a["idb"], a["dY"], a["lddy"], a["dW"], a["ldw"], a["n"], a["V"], a["D"], -1, 1.0,
                              None, a["ws"], a["nb"], None)


INV, ALIGN, NOMEM, LARGE = mp.MP_ERR_INVALID_ARG, mp.MP_ERR_ALIGNMENT, mp.MP_ERR_NOMEM, mp.MP_ERR_TOO_LARGE


def test_embedding_refusals(p16):
    L = mp.lib()
    for call in (_embed_fwd, _embed_bwd):
        assert call(L, p16, ids=None) == INV
        assert call(L, p16, n=-1) == INV and call(L, p16, V=0) == INV and call(L, p16, D=0) == INV
        assert call(L, p16, ldw=4) == INV and call(L, p16, ldw=12) == ALIGN
        assert call(L, p16, idb=2) == INV and call(L, p16, ids=p16 + 4) == ALIGN
    assert _embed_fwd(L, p16, Y=None) == INV and _embed_fwd(L, p16, W=p16 + 2) == ALIGN
    assert _embed_fwd(L, p16, ldy=4) == INV and _embed_fwd(L, p16, ldy=20) == ALIGN
    assert _embed_bwd(L, p16, dW=None) == INV and _embed_bwd(L, p16, dY=p16 + 8) == ALIGN
    assert _embed_bwd(L, p16, ws=None) == NOMEM and _embed_bwd(L, p16, ws=p16 + 4) == ALIGN
    need = mp.mp_embedding_bwd_workspace_bytes(4, 4, 8)
    assert need > 0 and _embed_bwd(L, p16, nb=need - 1) == NOMEM
    assert _embed_bwd(L, p16, n=(1 << 31) - 1) == LARGE and _embed_bwd(L, p16, V=1 << 31) == LARGE
    assert mp.mp_embedding_bwd_workspace_bytes(-1, 4, 8) == 0


def _norm_fwd(L, p, **k):
    a = dict(kind=0, eps=1e-6, x=p, xb=2, ldx=8, y=p, ldy=8, gpost=p, gate=p, ldgate=0, xo=p, ldxo=8, gpre=p, n=p, ldn=8,
             stats=p, M=4, D=8)
    a.update(k)
    return L.mp_block_norm_fwd(a["kind"], a["eps"], 1.0, a["x"], a["xb"], a["ldx"], a["y"], a["ldy"], a["gpost"], a["gate"],
                               a["ldgate"], a["xo"], a["ldxo"], a["gpre"], a["n"], a["ldn"], a["stats"], a["M"], a["D"],
                               None)


def _norm_bwd(L, p, **k):
    a = dict(kind=0, dn=p, lddn=8, up=p, ldup=8, xo=p, xb=2, ldxo=8, y=p, ldy=8, gpost=p, gate=p, ldgate=0, gpre=p, stats=p,
             dx=p, lddx=8, dy=p, lddy=8, dgpost=p, dgate=p, lddgate=0, dgpre=p, M=4, D=8, ws=p, nb=1 << 40)
    a.update(k)
    return L.mp_block_norm_bwd(a["kind"], 1.0, a["dn"], a["lddn"], a["up"], a["ldup"], a["xo"], a["xb"], a["ldxo"], a["y"],
                               a["ldy"], a["gpost"], a["gate"], a["ldgate"], a["gpre"], a["stats"], a["dx"], a["lddx"],
                               a["dy"], a["lddy"], a["dgpost"], a["dgate"], a["lddgate"], a["dgpre"], a["M"], a["D"], None,
                               a["ws"], a["nb"], None)


def test_block_norm_refusals(p16):
    L = mp.lib()
    for call in (_norm_fwd, _norm_bwd):
        assert call(L, p16, kind=2) == INV and call(L, p16, xb=8) == INV
        assert call(L, p16, M=-1) == INV and call(L, p16, D=0) == INV
        big = mp.MP_NORM_MAX_D + 8
        assert call(L, p16, D=big, ldx=big, ldn=big, ldxo=big, ldy=big, lddn=big, lddx=big, lddy=big, ldup=big) == LARGE
        assert call(L, p16, gpre=None) == INV and call(L, p16, y=None) == INV and call(L, p16, gpost=None) == INV
        assert call(L, p16, ldxo=4) == INV and call(L, p16, ldxo=12) == ALIGN
        assert call(L, p16, ldgate=4) == INV and call(L, p16, gate=p16 + 2) == ALIGN and call(L, p16, stats=p16 + 4) == ALIGN
    assert _norm_fwd(L, p16, eps=-1.0) == INV and _norm_fwd(L, p16, eps=float("nan")) == INV
    assert _norm_fwd(L, p16, x=None) == INV and _norm_fwd(L, p16, n=None) == INV and _norm_fwd(L, p16, xo=None) == INV
    assert _norm_fwd(L, p16, x=p16 + 2) == ALIGN and _norm_fwd(L, p16, ldn=12) == ALIGN
    # without a block there is no x_out and no gate
    assert _norm_fwd(L, p16, y=None, gpost=None, gate=None) == INV
    assert _norm_fwd(L, p16, y=None, gpost=None, xo=None) == INV
    assert _norm_bwd(L, p16, dgate=None) == INV and _norm_bwd(L, p16, gate=None) == INV
    assert _norm_bwd(L, p16, dy=None) == INV and _norm_bwd(L, p16, dgpost=None) == INV and _norm_bwd(L, p16, dgpre=None) == INV
    assert _norm_bwd(L, p16, stats=None) == INV and _norm_bwd(L, p16, dx=None) == INV and _norm_bwd(L, p16, dn=None) == INV
    assert _norm_bwd(L, p16, ldgate=8, lddgate=4) == INV and _norm_bwd(L, p16, ldgate=8, lddgate=12) == ALIGN
    assert _norm_bwd(L, p16, ldup=4) == INV and _norm_bwd(L, p16, ldup=12) == ALIGN
    assert _norm_bwd(L, p16, ws=None) == NOMEM and _norm_bwd(L, p16, ws=p16 + 8) == ALIGN
    need = mp.mp_block_norm_bwd_workspace_bytes(4, 8)
    assert need > 0 and _norm_bwd(L, p16, nb=need - 1) == NOMEM
    assert mp.mp_block_norm_bwd_workspace_bytes(4, mp.MP_NORM_MAX_D + 1) == 0
    # a result in an input's place has its pitch
    q = p16 + 1024
    apart = dict(x=q, y=q + 256, n=q + 512, xo=q + 768)
    for a, b in (("x", "xo"), ("y", "n")):
        assert _norm_fwd(L, p16, **{**apart, a: p16, b: p16, "ld" + b: 16}) == INV
    for a, b in (("up", "dx"), ("dn", "dy"), ("y", "dy")):
        k = dict(up=q, dn=q + 128, y=q + 256, dx=q + 384, dy=q + 512)
        assert _norm_bwd(L, p16, **{**k, a: p16, b: p16, "ld" + b: 16}) == INV
    assert _norm_bwd(L, p16, gate=p16, dgate=p16, ldgate=8, lddgate=16, dx=q, dy=q + 128) == INV
    # FP32 rows may start every 4 elements (M = 0: nothing is launched)
    assert _norm_fwd(L, p16, xb=4, ldx=12, ldxo=12, M=0) not in (INV, ALIGN)
    assert _norm_fwd(L, p16, xb=4, ldx=10, ldxo=12, M=0) == ALIGN


def _loss(L, p, cfg=(0.2, 0.2, 0.0, 1.0), **k):
    a = dict(z=p, ldl=8, t=p, idb=8, old=p, ref=p, adv=p, w=p, N=4, V=8, dz=p, lddl=8, lp=p, tl=p, loss=p)
    a.update(k)
    c = None if cfg is None else C.byref(mp.PolicyConfig(*cfg))
    return L.mp_policy_loss(a["z"], a["ldl"], a["t"], a["idb"], a["old"], a["ref"], a["adv"], a["w"], a["N"], a["V"], c,
                            a["dz"], a["lddl"], a["lp"], a["tl"], a["loss"], None, None)


def test_policy_loss_refusals(p16):
    L = mp.lib()
    assert _loss(L, p16, cfg=None) == INV
    for cfg in ((-0.1, 0.2, 0, 1), (0.2, -0.1, 0, 1), (0.2, 0.2, float("nan"), 1), (0.2, 0.2, 0, float("inf")),
                (float("nan"), 0.2, 0, 1)):
        assert _loss(L, p16, cfg=cfg) == INV
    for name in ("z", "t", "old", "adv", "w", "lp", "tl"):
        assert _loss(L, p16, **{name: None}) == INV
    assert _loss(L, p16, N=-1) == INV and _loss(L, p16, V=0) == INV and _loss(L, p16, idb=3) == INV
    big = 524288 + 8
    assert _loss(L, p16, V=big, ldl=big, lddl=big) == LARGE
    assert _loss(L, p16, dz=p16, lddl=16) == INV
    assert _loss(L, p16, ldl=4) == INV and _loss(L, p16, lddl=4) == INV
    assert _loss(L, p16, ldl=12) == ALIGN and _loss(L, p16, lddl=12) == ALIGN
    assert _loss(L, p16, z=p16 + 2) == ALIGN and _loss(L, p16, t=p16 + 4) == ALIGN and _loss(L, p16, adv=p16 + 2) == ALIGN
    assert L.mp_token_logp(p16, 8, p16, 8, None, 4, 8, None, None, None) == INV
    assert L.mp_token_logp(p16, 8, p16, 8, None, 4, 9, p16, None, None) == INV
    assert L.mp_token_logp(p16, 12, p16, 8, None, 4, 8, p16, None, None) == ALIGN


def _plan(L, p, **k):
    a = dict(n=1, g=p, w=p, m=p, v=p, w16=p, count=8, decay=1.0, bits=32, ms=None, vs=None, out=True)
    a.update(k)
    arr = lambda x: None if x is None else (C.c_void_p * 1)(x or None)  # noqa: E731
    out = C.c_void_p()
    return L.mp_adamw_plan_create(a["n"], arr(a["g"]), arr(a["w"]), arr(a["m"]), arr(a["v"]), arr(a["w16"]),
                                  (C.c_int64 * 1)(a["count"]), (C.c_float * 1)(a["decay"]), a["bits"], arr(a["ms"]),
                                  arr(a["vs"]), C.byref(out) if a["out"] else None)


def test_adamw_refusals(p16):
    L = mp.lib()
    assert _plan(L, p16, n=0) == INV and _plan(L, p16, out=False) == INV and _plan(L, p16, count=-1) == INV
    for name in ("g", "w", "m", "v", "w16"):
        assert _plan(L, p16, **{name: None}) == INV and _plan(L, p16, **{name: 0}) == INV
        assert _plan(L, p16, **{name: p16 + 4}) == ALIGN
    assert _plan(L, p16, decay=float("nan")) == INV
    assert _plan(L, p16, bits=16) == INV and _plan(L, p16, bits=8) == INV and _plan(L, p16, ms=p16, vs=p16) == INV
    assert _plan(L, p16, bits=8, ms=p16) == INV and _plan(L, p16, bits=8, ms=p16, vs=0) == INV
    assert _plan(L, p16, bits=8, ms=p16 + 2, vs=p16) == ALIGN
    assert L.mp_adamw_update(None, None, None, 0, None) == INV
    assert L.mp_adamw_plan_destroy(None) == mp.MP_OK
