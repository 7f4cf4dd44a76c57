"""Head norms without an eps, where the heads do not fill a warp's last round.  Tolerances as in the file of the cases."""
import pytest
import torch

import test_gpu_head_norm as heads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [dict(T=50, hq=5, hk=3, D=64, rot=64), dict(T=33, hq=7, hk=1, D=128, rot=64), dict(T=20, hq=25, hk=5, D=128, rot=128),
                               dict(T=9, hq=1, hk=1, D=8, rot=0), dict(T=70, hq=3, hk=0, D=24, rot=16, pairs=True),
                               dict(T=4000, hq=0, hk=3, D=40, rot=32), dict(T=30, hq=2, hk=1, D=256, rot=256)],
                         ids=lambda k: "-".join(str(v) for v in k.values()))
def test_no_eps(mp, monkeypatch, k):
    monkeypatch.setattr(heads, "EPS", 0.0)
    c = heads.Case(**k)
    c.x[:] = torch.where(c.x.abs() < 0.01, 0.5, c.x)          # no head is 0
    y, dx = (torch.empty(c.x.shape, dtype=torch.float16, device="cuda") for _ in "yd")
    dg = [torch.full((c.D,), 7.0, dtype=torch.float16, device="cuda") for _ in "qk"]
    ws = torch.empty(mp.mp_head_norm_rope_bwd_workspace_bytes(c.T, c.hq, c.hk, c.D), dtype=torch.uint8, device="cuda")
    st = mp.State(8.0)
    mp.mp_head_norm_rope_fwd(c.x, c.gq, c.gk, c.pos, c.freqs, y, c.hq, c.hk, eps=0.0, pairs=c.pairs)
    mp.mp_head_norm_rope_bwd(c.dy, c.x, c.gq, c.gk, c.pos, c.freqs, dx, *dg, c.hq, c.hk, eps=0.0, pairs=c.pairs, state=st, workspace=ws)
    c.check_forward(y)
    c.check_backward(dx, *dg)
    assert st.read().found_inf == 0
