"""Refusals of the calls that mix tokens and learn from a teacher: every bad argument is found on the host, before any CUDA call."""
import ctypes as C

import pytest
import torch

from paper_1805_10387_b200 import mp

_BUF = (C.c_uint16 * 8192)()
INV, ALIGN, NOMEM, LARGE = mp.MP_ERR_INVALID_ARG, mp.MP_ERR_ALIGNMENT, mp.MP_ERR_NOMEM, mp.MP_ERR_TOO_LARGE


@pytest.fixture
def p16():
    """A 16-byte aligned host address: no call of this file gets as far as reading it."""
    return (C.addressof(_BUF) + 15) // 16 * 16


def _heads_fwd(L, p, **k):
    a = dict(x=p, ldx=192, gq=p, gk=p, pos=p, pb=8, f=p, rot=32, pairs=0, eps=1e-6, y=p, ldy=192, T=4, hq=2, hk=1, D=64)
    a.update(k)
    return L.mp_head_norm_rope_fwd(*(a[n] for n in ("x", "ldx", "gq", "gk", "pos", "pb", "f", "rot", "pairs", "eps", "y", "ldy", "T",
                                                    "hq", "hk", "D")), None)


def _heads_bwd(L, p, **k):
    a = dict(dy=p, lddy=192, x=p, ldx=192, gq=p, gk=p, pos=p, pb=8, f=p, rot=32, pairs=0, eps=1e-6, y=p, ldy=192, dgq=p, dgk=p, T=4,
             hq=2, hk=1, D=64, ws=p, nb=1 << 40)
    a.update(k)
    return L.mp_head_norm_rope_bwd(*(a[n] for n in ("dy", "lddy", "x", "ldx", "gq", "gk", "pos", "pb", "f", "rot", "pairs", "eps", "y",
                                                    "ldy", "dgq", "dgk", "T", "hq", "hk", "D")), None, a["ws"], a["nb"], None)


def test_head_norm_refusals(p16):
    L = mp.lib()
    for call in (_heads_fwd, _heads_bwd):
        for bad in (dict(T=-1), dict(hq=-1), dict(hq=0, hk=0), dict(D=0), dict(D=60), dict(rot=-16), dict(rot=24), dict(rot=80),
                    dict(pairs=2), dict(eps=-1.0), dict(eps=float("nan")), dict(pb=2), dict(ldx=184), dict(ldy=184), dict(x=None),
                    dict(y=None), dict(pos=None), dict(f=None)):
            assert call(L, p16, **bad) == INV, bad
        for bad in (dict(ldx=196), dict(ldy=196), dict(x=p16 + 2), dict(y=p16 + 8), dict(gq=p16 + 2), dict(gk=p16 + 2),
                    dict(pos=p16 + 4), dict(f=p16 + 4)):
            assert call(L, p16, **bad) == ALIGN, bad
        big = mp.MP_HEAD_MAX_D + 8
        assert call(L, p16, D=big, ldx=3 * big, ldy=3 * big, lddy=3 * big) == LARGE if call is _heads_bwd else \
            call(L, p16, D=big, ldx=3 * big, ldy=3 * big) == LARGE
        assert call(L, p16, x=p16, y=p16, ldy=200) == INV
        # without a rotation there are no positions
        assert call(L, p16, rot=0, pos=None, f=None, pb=0, T=0) not in (INV, ALIGN)
    assert _heads_bwd(L, p16, dy=None) == INV and _heads_bwd(L, p16, lddy=184) == INV and _heads_bwd(L, p16, lddy=196) == ALIGN
    assert _heads_bwd(L, p16, dgq=None) == INV and _heads_bwd(L, p16, gk=None) == INV and _heads_bwd(L, p16, gk=None, dgk=None) == INV
    assert _heads_bwd(L, p16, dgk=p16 + 2) == ALIGN and _heads_bwd(L, p16, ws=p16 + 8) == ALIGN
    assert _heads_bwd(L, p16, x=p16 + 1024, y=p16, dy=p16, ldy=200) == INV
    need = mp.mp_head_norm_rope_bwd_workspace_bytes(4, 2, 1, 64)
    assert need > 0 and _heads_bwd(L, p16, nb=need - 1) == NOMEM and _heads_bwd(L, p16, ws=None) == NOMEM
    assert mp.mp_head_norm_rope_bwd_workspace_bytes(4, 2, 1, 60) == 0


def _attn(L, p, bwd=False, **k):
    a = dict(do=p, q=p, k=p, v=p, o=p, dq=p, dk=p, dv=p, lse=p, off=p, ob=4, n=2, T=64, hq=4, hk=2, D=32, scale=0.2, causal=1, window=0,
             ws=p, nb=1 << 40)
    a.update({"ld" + x: 128 if x in ("do", "q", "o", "dq") else 64 for x in ("do", "q", "k", "v", "o", "dq", "dk", "dv")})
    a.update(k)
    m = lambda *names: [v for x in names for v in (a[x], a["ld" + x])]  # noqa: E731
    tail = [a["off"], a["ob"], a["n"], a["T"], a["hq"], a["hk"], a["D"], a["scale"], a["causal"], a["window"], None]
    if bwd:
        return L.mp_attention_bwd(*m("do", "q", "k", "v", "o"), a["lse"], *m("dq", "dk", "dv"), *tail, a["ws"], a["nb"], None)
    return L.mp_attention_fwd(*m("q", "k", "v", "o"), a["lse"], *tail, None)


def test_attention_refusals(p16):
    L = mp.lib()
    for bwd in (False, True):
        for bad in (dict(n=-1), dict(T=-1), dict(hq=0), dict(hk=0), dict(hk=3), dict(D=0), dict(D=30), dict(ob=2), dict(scale=0.0),
                    dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(causal=2), dict(window=-1),
                    dict(window=5, causal=0), dict(off=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None),
                    dict(ldq=120), dict(ldk=56), dict(ldv=56), dict(ldo=120)):
            assert _attn(L, p16, bwd, **bad) == INV, bad
        for bad in (dict(q=p16 + 2), dict(k=p16 + 8), dict(v=p16 + 2), dict(o=p16 + 2), dict(ldq=132), dict(ldv=68), dict(lse=p16 + 2),
                    dict(off=p16 + 2), dict(off=p16 + 4, ob=8)):
            assert _attn(L, p16, bwd, **bad) == ALIGN, bad
        big = dict(D=mp.MP_ATTENTION_MAX_D + 8)
        big.update({"ld" + x: 4096 for x in ("do", "q", "k", "v", "o", "dq", "dk", "dv")})
        assert _attn(L, p16, bwd, **big) == LARGE
        assert _attn(L, p16, bwd, T=mp.MP_ATTENTION_MAX_ROWS + 1) == LARGE
        assert _attn(L, p16, bwd, n=1 << 29) == LARGE
    for bad in (dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(lddq=120), dict(lddk=56)):
        assert _attn(L, p16, True, **bad) == INV, bad
    assert _attn(L, p16, True, lddv=68) == ALIGN and _attn(L, p16, True, dk=p16 + 2) == ALIGN and _attn(L, p16, True, ws=p16 + 8) == ALIGN
    need = mp.mp_attention_bwd_workspace_bytes(64, 4, 2, 32)
    assert need > 0 and _attn(L, p16, True, nb=need - 1) == NOMEM and _attn(L, p16, True, ws=None) == NOMEM
    assert mp.mp_attention_bwd_workspace_bytes(64, 4, 3, 32) == 0


def test_attention_refuses_results_in_an_inputs_place(p16):
    L, at = mp.lib(), {x: p16 + 1024 * i for i, x in enumerate(("do", "q", "k", "v", "o", "dq", "dk", "dv"))}
    for x in ("q", "k", "v"):
        assert _attn(L, p16, **{**at, "o": at[x]}) == INV
    for x in ("dq", "dk", "dv"):
        for y in at:
            assert x == y or _attn(L, p16, True, **{**at, x: at[y]}) == INV, (x, y)
    q = torch.zeros(4, 0, dtype=torch.float16)
    with pytest.raises(ValueError):
        mp.mp_attention_fwd(q, q, q, q, torch.zeros(1, 4), torch.zeros(2, dtype=torch.int32), 1, 1)


def _top(L, p, **k):
    a = dict(z=p, ldl=64, t=p, tb=8, w=p, N=4, V=60, k=5, temp=1.0, lp=p, ent=p, ids=p, tlp=p)
    a.update(k)
    return L.mp_token_top(*(a[n] for n in ("z", "ldl", "t", "tb", "w", "N", "V", "k", "temp", "lp", "ent", "ids", "tlp")), None, None)


def test_token_top_refusals(p16):
    L = mp.lib()
    for bad in (dict(N=-1), dict(V=0), dict(k=0), dict(k=61), dict(ldl=56), dict(tb=3), dict(temp=0.0), dict(temp=1e4), dict(temp=float("nan")),
                dict(z=None), dict(ids=None), dict(tlp=None), dict(t=None), dict(lp=None)):
        assert _top(L, p16, **bad) == INV, bad
    for bad in (dict(ldl=68), dict(z=p16 + 2), dict(t=p16 + 4), dict(ids=p16 + 2), dict(tlp=p16 + 1), dict(w=p16 + 2), dict(ent=p16 + 2)):
        assert _top(L, p16, **bad) == ALIGN, bad
    big = 524288 + 8
    assert _top(L, p16, V=big, ldl=big) == LARGE and _top(L, p16, V=1000, ldl=1000, k=mp.MP_TOP_MAX_K + 1) == LARGE
    assert _top(L, p16, N=1 << 27) == LARGE


def _distill(L, p, cfg=(1.0, 1, 1.0), **k):
    a = dict(z=p, ldl=64, ids=p, ib=8, tlp=p, K=5, w=p, N=4, V=60, dz=p, lddl=64, tl=p, loss=p)
    a.update(k)
    c = None if cfg is None else C.byref(mp.DistillConfig(*cfg))
    return L.mp_distill_loss(*(a[n] for n in ("z", "ldl", "ids", "ib", "tlp", "K", "w", "N", "V")), c,
                             *(a[n] for n in ("dz", "lddl", "tl", "loss")), None, None)


def test_distill_refusals(p16):
    L = mp.lib()
    for cfg in (None, (0.0, 1, 1.0), (1e4, 1, 1.0), (float("nan"), 1, 1.0), (1.0, 2, 1.0), (1.0, 1, float("inf"))):
        assert _distill(L, p16, cfg) == INV, cfg
    for bad in (dict(N=-1), dict(V=0), dict(K=0), dict(K=61), dict(ldl=56), dict(lddl=56), dict(ib=2), dict(z=None), dict(ids=None),
                dict(tlp=None), dict(w=None), dict(tl=None), dict(lddl=72)):
        assert _distill(L, p16, **bad) == INV, bad
    for bad in (dict(ldl=68, dz=p16 + 1024), dict(lddl=68, dz=p16 + 1024), dict(z=p16 + 2), dict(ids=p16 + 4), dict(tlp=p16 + 2),
                dict(loss=p16 + 2)):
        assert _distill(L, p16, **bad) == ALIGN, bad
    big = 524288 + 8
    assert _distill(L, p16, V=big, ldl=big, lddl=big) == LARGE
    assert _distill(L, p16, V=1000, ldl=1000, lddl=1000, K=mp.MP_DISTILL_MAX_K + 1) == LARGE


def test_the_binding_refuses_what_is_not_on_the_device_or_misshapen():
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)  # noqa: E731
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        mp.mp_attention_fwd(h(8, 64), h(8, 64), h(8, 64), h(8, 64), torch.zeros(1, 8), i, 1, 1)
    with pytest.raises(ValueError):
        mp.mp_attention_fwd(h(8, 64), h(8, 64), h(8, 64), h(8, 64), torch.zeros(1, 8), i, 3, 1)
    with pytest.raises(ValueError):
        mp.mp_head_norm_rope_fwd(h(8, 64), None, None, None, None, h(8, 64), 2, 1)
    with pytest.raises(TypeError):
        mp.mp_token_top(h(8, 64), torch.zeros(8, 4, dtype=torch.int32), torch.zeros(8, 4))
    with pytest.raises(TypeError):
        mp.mp_distill_loss(h(8, 64), torch.zeros(8, 4, dtype=torch.int32), torch.zeros(8, 4), torch.ones(8), torch.ones(8))
