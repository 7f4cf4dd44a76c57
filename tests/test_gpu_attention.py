"""Attention over packed sequences against its formula in 64 bits.

Tolerances, from the roundings: a weight p enters its product in FP16 (half a step: 2^-11 of it, 2^-25 where it is subnormal;
the largest of a row is at least 1 then, and so is the sum), an output is rounded once (2^-11 of it), a score is an FP32
sum of D products (at most D 2^-24 of the sum of their magnitudes, and as much again for its exponent).  Backward: p
(2^-11, or 2^-37 where its 2^12 fold is subnormal) and ds (2^-11, or 2^-39 of its bound) enter in FP16, and what o, lse and the
scores are off by enters through them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

H = 2.0 ** -11


def _pad(n):
    return -(-n // 8) * 8


def _mat(g, rows, cols, std=1.0, extra=0):
    """Columns of a wider buffer, its other columns NaN."""
    full = torch.full((rows, _pad(cols) + extra), float("nan"), dtype=torch.float16, device="cuda")
    full[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std
    return full[:, :cols]


class Case:
    def __init__(self, lengths, hq, hk, D, causal=True, window=0, seed=0, before=0, after=0, std=1.0, scale=None, wide=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lengths, self.hq, self.hk, self.D, self.causal, self.window = lengths, hq, hk, D, causal, window
        self.before = before
        self.T = T = before + sum(lengths) + after
        self.scale = D ** -0.5 if scale is None else scale
        at = [before]
        for n in lengths:
            at.append(at[-1] + n)
        self.offsets = torch.tensor(at, dtype=torch.int64 if wide else torch.int32, device="cuda")
        self.q, self.k = _mat(g, T, hq * D, std, 8), _mat(g, T, hk * D, std)
        self.v, self.do = _mat(g, T, hk * D, std, 24), _mat(g, T, hq * D, 0.5)
        for t in (self.q, self.k, self.v, self.do):          # rows of no sequence do not matter
            t[:before] = float("nan")
            t[before + sum(lengths):] = float("inf")
        self.o = torch.full((T, hq * D + 16), 7.0, dtype=torch.float16, device="cuda")[:, :hq * D]
        self.lse = torch.full((hq, T), 7.0, device="cuda")

    def forward(self, mp, **k):
        mp.mp_attention_fwd(self.q, self.k, self.v, self.o, self.lse, self.offsets, self.hq, self.hk, scale=self.scale,
                            causal=self.causal, window=self.window, **k)

    def backward(self, mp, **k):
        wide, narrow = (self.T, self.hq * self.D), (self.T, self.hk * self.D)
        self.grads = [torch.full((r, c + 8), 7.0, dtype=torch.float16, device="cuda")[:, :c] for r, c in (wide, narrow, narrow)]
        if "workspace" not in k:
            need = mp.mp_attention_bwd_workspace_bytes(self.T, self.hq, self.hk, self.D)
            k["workspace"] = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        mp.mp_attention_bwd(self.do, self.q, self.k, self.v, self.o, self.lse, *self.grads, self.offsets, self.hq, self.hk,
                            scale=self.scale, causal=self.causal, window=self.window, **k)

    def parts(self):
        at = self.before
        for n in self.lengths:
            r = slice(at, at + n)
            at += n
            if n == 0:
                continue
            i = torch.arange(n, device="cuda")
            seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
            if self.causal:
                seen &= i[None] <= i[:, None]
                if self.window:
                    seen &= i[:, None] - i[None] < self.window
            for h in range(self.hq):
                c = h * self.hk // self.hq
                yield r, h, slice(h * self.D, (h + 1) * self.D), slice(c * self.D, (c + 1) * self.D), seen

    def check_forward(self):
        for r, h, a, b, seen in self.parts():
            q, k, v = self.q[r, a].double(), self.k[r, b].double(), self.v[r, b].double()
            x = (q @ k.T * self.scale).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(x, 1)
            p = (x - lse[:, None]).exp()
            es = (q.abs() @ k.abs().T).masked_fill(~seen, 0).amax(1, keepdim=True) * self.scale * self.D * 2.0 ** -23 + 2.0 ** -20
            o, mag = p @ v, p @ v.abs()
            tol = H * (mag + o.abs()) * 1.01 + 2 * es * mag + 2.0 ** -25 * (seen.double() @ v.abs()) + 2.0 ** -25
            err = (self.o[r, a].double() - o).abs()
            assert bool((err <= tol).all()), (r, h, (err / tol).max().item())
            err = (self.lse[h, r].double() - lse).abs()
            assert bool((err <= es[:, 0] + 2.0 ** -22 * lse.abs()).all()), (r, h, err.max().item())

    def check_backward(self):
        dq, dk, dv = self.grads
        at = {}
        bound = 0.0
        for r, h, a, b, seen in self.parts():
            bound = max(bound, 2 * (self.do[r, a].double().norm(dim=1).max() * self.v[r, b].double().norm(dim=1).max()).item())
        for r, h, a, b, seen in self.parts():
            q, k, v, do = self.q[r, a].double(), self.k[r, b].double(), self.v[r, b].double(), self.do[r, a].double()
            x = (q @ k.T * self.scale).masked_fill(~seen, -math.inf)
            p = torch.softmax(x, 1)
            o = p @ v
            es = (q.abs() @ k.abs().T).masked_fill(~seen, 0).amax(1, keepdim=True) * self.scale * self.D * 2.0 ** -22 + 2.0 ** -19
            dp, delta = do @ v.T, (do * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            off = (do.abs() * (self.o[r, a].double() - o).abs()).sum(1, keepdim=True)          # what o's rounding does to delta
            small = self.D * 2.0 ** -23 * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))
            e_p = p * (H * 1.01 + 2 * es) + 2.0 ** -37 * seen
            e_ds = ds.abs() * H * 1.01 + 2 * es * p * (dp - delta).abs() + p * (off + small) * 1.01 + 2.0 ** -38 * bound * seen
            got, want = dq[r, a].double(), self.scale * (ds @ k)
            tol = self.scale * (e_ds @ k.abs()) + H * want.abs() * 1.01 + 2.0 ** -25
            assert bool(((got - want).abs() <= tol).all()), ("dq", r, h, ((got - want).abs() / tol).max().item())
            part = at.setdefault((r.start, b.start), [r, b, 0, 0, 0, 0])
            part[2] = part[2] + self.scale * (ds.T @ q)
            part[3] = part[3] + self.scale * (e_ds.T @ q.abs())
            part[4] = part[4] + p.T @ do
            part[5] = part[5] + e_p.T @ do.abs()
        for r, b, k, ek, v, ev in at.values():
            for name, got, want, e in (("dk", dk, k, ek), ("dv", dv, v, ev)):
                tol = e + H * want.abs() * 1.01 + 2.0 ** -25
                err = (got[r, b].double() - want).abs()
                assert bool((err <= tol).all()), (name, r, b, (err / tol).max().item())
        end = self.before + sum(self.lengths)
        for t in self.grads:
            assert bool((t[:self.before] == 7.0).all()) and bool((t[end:] == 7.0).all())
            assert bool((t.as_strided((self.T, 8), t.stride(), t.shape[1]) == 7.0).all())

    def check_untouched(self):
        end = self.before + sum(self.lengths)
        for t in (self.o[:self.before], self.o[end:], self.lse[:, :self.before], self.lse[:, end:], self.o.as_strided(
                (self.T, 16), self.o.stride(), self.hq * self.D)):
            assert bool((t == 7.0).all())


SHAPES = [
    ([1], 1, 1, 64), ([37], 2, 2, 64), ([128], 2, 1, 128), ([129], 1, 1, 128), ([256, 257, 255], 2, 2, 64),
    ([0, 1, 127, 0, 128, 2, 385, 0], 4, 2, 128), ([300, 700], 3, 3, 40), ([513], 2, 2, 8), ([200, 31], 6, 2, 72),
    ([640], 2, 1, 96), ([1000], 8, 1, 16), ([65] * 9, 2, 2, 120),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,hq,hk,D", SHAPES)
def test_forward(mp, lengths, hq, hk, D, causal):
    c = Case(lengths, hq, hk, D, causal, before=3 if len(lengths) > 1 else 0, after=5 if D != 64 else 0, wide=hq == 2)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()


@pytest.mark.parametrize("window", [1, 2, 127, 128, 129, 300, 5000])
def test_forward_window(mp, window):
    c = Case([700, 3, 260], 2, 1, 64, window=window)
    c.forward(mp)
    c.check_forward()


@pytest.mark.parametrize("std,scale", [(8.0, 1.0), (0.01, 0.05), (30.0, 0.2)])
def test_forward_of_sharp_and_flat_rows(mp, std, scale):
    c = Case([600], 2, 2, 64, std=std, scale=scale)
    c.forward(mp)
    c.check_forward()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,hq,hk,D", SHAPES)
def test_backward(mp, lengths, hq, hk, D, causal):
    c = Case(lengths, hq, hk, D, causal, before=3 if len(lengths) > 1 else 0, after=5 if D != 64 else 0, wide=hq == 2)
    c.forward(mp)
    c.backward(mp)
    c.check_backward()


@pytest.mark.parametrize("window", [1, 2, 127, 128, 129, 300, 5000])
def test_backward_window(mp, window):
    c = Case([700, 3, 260], 2, 1, 64, window=window)
    c.forward(mp)
    c.backward(mp)
    c.check_backward()


@pytest.mark.parametrize("std,scale", [(8.0, 1.0), (0.01, 0.05), (30.0, 0.2)])
def test_backward_of_sharp_and_flat_rows(mp, std, scale):
    c = Case([600], 2, 2, 64, std=std, scale=scale)
    c.forward(mp)
    c.backward(mp)
    c.check_backward()


@pytest.mark.parametrize("window", [0, 1, 31, 33, 65, 129, 700])
@pytest.mark.parametrize("lengths", [[512], [513], [1500], [1, 0, 1023], [0, 0, 0, 1300, 31, 33], [511, 513, 515], [97, 1700]])
@pytest.mark.parametrize("D", [64, 40])
def test_forward_windows_of_many_lengths(mp, D, lengths, window):
    c = Case(lengths, 2, 1, D, window=window, seed=len(lengths) + window)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()


@pytest.mark.parametrize("lengths", [[513], [1500], [129, 1, 31, 33, 65, 96], [1300, 97]])
@pytest.mark.parametrize("D", [64, 8])
def test_forward_of_all_keys_many_lengths(mp, D, lengths):
    c = Case(lengths, 2, 2, D, causal=False, seed=D, before=3, after=5)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()
