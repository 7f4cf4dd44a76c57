"""What the token model refuses when it is made, before it asks for any memory of the device."""
import pytest

from paper_1805_10387_b200 import mp
from paper_1805_10387_b200.token_model import TokenModel


class Reached(Exception):
    pass


@pytest.mark.parametrize("k", [dict(head_dim=mp.MP_ATTENTION_MAX_D + 8), dict(head_dim=256), dict(head_dim=60), dict(head_dim=0), dict(head_dim=-8),
                               dict(heads=3, kv_heads=2), dict(kv_heads=0), dict(kv_heads=-1), dict(heads=-2), dict(window=-1),
                               dict(sequences=0)], ids=str)
def test_refusals(monkeypatch, k):
    def state(*a):
        raise Reached
    monkeypatch.setattr(mp, "State", state)
    with pytest.raises(ValueError):
        TokenModel(40, 32, 64, 1, 16, **{"heads": 2, **k})


@pytest.mark.parametrize("k", [dict(heads=2, head_dim=mp.MP_ATTENTION_MAX_D), dict(heads=6, kv_heads=3, head_dim=8, window=5),
                               dict(heads=0, head_dim=256, kv_heads=5)], ids=str)
def test_what_is_taken(monkeypatch, k):
    def state(*a):
        raise Reached
    monkeypatch.setattr(mp, "State", state)
    with pytest.raises(Reached):
        TokenModel(40, 32, 64, 1, 16, **k)
