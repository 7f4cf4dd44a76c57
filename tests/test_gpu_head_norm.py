"""Norms of queries and keys for each head with the position rotation, against the formulas in 64 bits.

Tolerances: sums of at most 256 squares, a reciprocal root and a cosine in FP32 are off by less than 2^-19 of the magnitudes that
meet in an output; that output is rounded once to FP16 (2^-11 of it; 2^-25 where it is subnormal)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

H, F = 2.0 ** -11 * 1.001, 2.0 ** -19
EPS = 1e-6


def _mat(g, rows, cols, std=1.0, extra=8):
    full = torch.full((rows, -(-cols // 8) * 8 + extra), float("nan"), dtype=torch.float16, device="cuda")
    full[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std
    return full[:, :cols]


def _turned(x, pos, freqs, pairs, back=False):
    """x [T, heads, D] in 64 bits; angles reduced with whole turns taken off exactly."""
    rot = 2 * len(freqs)
    if rot == 0:
        return x
    t = torch.tensor([[(int(p) * float(f)) if abs(int(p)) < 2 ** 20 else float(_mod_turn(int(p), float(f))) for f in freqs.tolist()]
                      for p in pos.tolist()], dtype=torch.float64, device=x.device)[:, None]
    c, s = t.cos(), t.sin() * (-1 if back else 1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, a * s + b * c
    turned = torch.stack([u, v], 3).flatten(2) if pairs else torch.cat([u, v], 2)
    return torch.cat([turned, x[..., rot:]], 2)


def _mod_turn(p, f):
    """p f modulo a turn, in radians, with a long pi."""
    from fractions import Fraction
    pi2 = Fraction(62831853071795864769252867665590057683943387987502, 10 ** 49)
    a = Fraction(p) * Fraction(f)
    return float(a - pi2 * (a // pi2))


class Case:
    def __init__(self, T, hq, hk, D, rot, pairs=False, gains=True, start=0, wide=True, seed=0, std=1.5):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.hq, self.hk, self.D, self.pairs = T, hq, hk, D, pairs
        self.x = _mat(g, T, (hq + hk) * D, std, extra=hk * D)        # values follow in the row
        self.dy = _mat(g, T, (hq + hk) * D)
        self.gq, self.gk = ((1 + 0.3 * torch.randn(D, generator=g, device="cuda")).half() for _ in "qk") if gains else (None, None)
        self.pos = (start + torch.arange(T, device="cuda") * 3).to(torch.int64 if wide else torch.int32)
        self.freqs = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None

    def exact(self):
        x = self.x.double().reshape(self.T, -1, self.D)
        root = 1 / torch.sqrt((x * x).mean(2, keepdim=True) + EPS)
        one = torch.ones(self.D, dtype=torch.float64, device="cuda")
        gain = torch.cat([(one if self.gq is None else self.gq.double()).expand(self.hq, -1),
                          (one if self.gk is None else self.gk.double()).expand(self.hk, -1)])
        return x, root, gain

    def turn(self, v, back=False):
        return _turned(v, self.pos, self.freqs if self.freqs is not None else [], self.pairs, back)

    def check_forward(self, y):
        x, root, gain = self.exact()
        n = x * root * gain
        want = self.turn(n).reshape(self.T, -1)
        reach = n.abs().amax(2, keepdim=True).expand_as(n).reshape(self.T, -1)
        err = (y.double() - want).abs()
        assert bool((err <= H * want.abs() + 2 * F * reach + 2.0 ** -25).all()), (err - H * want.abs()).max().item()

    def check_backward(self, dx, dgq, dgk):
        x, root, gain = self.exact()
        u = self.turn(self.dy.double().reshape(self.T, -1, self.D), back=True)
        hat = x * root
        d = u * gain
        want = ((d - hat * (d * hat).mean(2, keepdim=True)) * root).reshape(self.T, -1)
        reach = ((d.abs().amax(2, keepdim=True) + hat.abs() * (d * hat).abs().mean(2, keepdim=True)) * root).reshape(self.T, -1)
        err = (dx.double() - want).abs()
        assert bool((err <= H * want.abs() + 4 * F * reach + 2.0 ** -25).all()), (err - H * want.abs()).max().item()
        if self.gq is not None:
            ug = u * hat
            near = u.abs().amax(2, keepdim=True) * hat.abs()          # a turned gradient is off by that much
            for got, part, mag in ((dgq, ug[:, :self.hq], near[:, :self.hq]), (dgk, ug[:, self.hq:], near[:, self.hq:])):
                want, tol = part.sum((0, 1)), mag.sum((0, 1)) * 4 * F
                err = (got.double() - want).abs()
                assert bool((err <= H * want.abs() + tol + 2.0 ** -25).all()), (err / (H * want.abs() + tol)).max().item()


CASES = [
    dict(T=1, hq=1, hk=1, D=64, rot=64), dict(T=16, hq=16, hk=4, D=64, rot=64, start=900_000), dict(T=33, hq=5, hk=1, D=8, rot=0),
    dict(T=100, hq=3, hk=3, D=80, rot=80, pairs=True), dict(T=77, hq=7, hk=2, D=128, rot=64, wide=False),
    dict(T=50, hq=9, hk=3, D=256, rot=256), dict(T=50, hq=2, hk=2, D=200, rot=96, pairs=True), dict(T=64, hq=0, hk=3, D=32, rot=32),
    dict(T=64, hq=3, hk=0, D=40, rot=32), dict(T=700, hq=4, hk=2, D=24, rot=16, gains=False), dict(T=9000, hq=2, hk=1, D=16, rot=16),
    dict(T=3, hq=70, hk=33, D=64, rot=32), dict(T=40, hq=2, hk=2, D=128, rot=128, start=-60),
    dict(T=40, hq=2, hk=2, D=64, rot=64, start=2 ** 31 - 200), dict(T=20, hq=1, hk=1, D=64, rot=64, start=2 ** 33),
]


@pytest.mark.parametrize("k", CASES, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_forward(mp, k):
    c = Case(**k)
    y = torch.full((c.T, c.x.shape[1] + 8), 7.0, dtype=torch.float16, device="cuda")
    mp.mp_head_norm_rope_fwd(c.x, c.gq, c.gk, c.pos, c.freqs, y[:, :-8], c.hq, c.hk, eps=EPS, pairs=c.pairs)
    c.check_forward(y[:, :-8])
    assert bool((y[:, -8:] == 7.0).all())
    # in the input's place: the same bits, and what follows in the row stays
    whole = c.x.as_strided((c.T, c.x.stride(0) if c.T > 1 else c.x.shape[1]), (c.x.stride(0), 1))
    rest = whole[:, c.x.shape[1]:].clone()
    mp.mp_head_norm_rope_fwd(c.x, c.gq, c.gk, c.pos, c.freqs, c.x, c.hq, c.hk, eps=EPS, pairs=c.pairs)
    assert torch.equal(c.x, y[:, :-8])
    assert torch.equal(whole[:, c.x.shape[1]:].view(torch.int16), rest.view(torch.int16))


@pytest.mark.parametrize("k", CASES, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_backward(mp, k):
    c = Case(**k)
    dx = torch.full((c.T, c.x.shape[1] + 8), 7.0, dtype=torch.float16, device="cuda")
    dgq, dgk = (None, None) if c.gq is None else (torch.full((c.D,), 7.0, dtype=torch.float16, device="cuda") for _ in "qk")
    need = mp.mp_head_norm_rope_bwd_workspace_bytes(c.T, c.hq, c.hk, c.D)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    call = lambda out, a, b: mp.mp_head_norm_rope_bwd(c.dy, c.x, c.gq, c.gk, c.pos, c.freqs, out, a, b, c.hq, c.hk, eps=EPS,  # noqa: E731
                                                      pairs=c.pairs, workspace=ws)
    call(dx[:, :-8], dgq, dgk)
    c.check_backward(dx[:, :-8], dgq, dgk)
    assert bool((dx[:, -8:] == 7.0).all())
    again = [None if t is None else torch.empty_like(t) for t in (dgq, dgk)]
    call(c.dy, *again)                                       # in the gradient's place, the same bits
    assert torch.equal(c.dy, dx[:, :-8])
    assert all(a is None or torch.equal(a, b) for a, b in zip(again, (dgq, dgk)))
