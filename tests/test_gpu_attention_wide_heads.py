"""Attention with heads of more than 64 elements (two tiles of queries share a block's keys there): windows, sharp and flat rows, many
lengths, and the long sequences that the other files leave to narrow heads.  Tolerances as in the files that the checks come from."""
import pytest
import torch

from test_gpu_attention import Case
from test_gpu_attention_edges import check_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [1, 2, 65, 127, 128, 129, 255, 256, 257, 300, 5000])
@pytest.mark.parametrize("D", [72, 128])
def test_windows_forward_and_backward(mp, D, window):
    c = Case([700, 3, 260, 0, 257], 2, 1, D, window=window, before=3, after=5, seed=window)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()
    c.backward(mp)
    c.check_backward()


@pytest.mark.parametrize("window", [0, 1, 31, 65, 129, 300, 700])
@pytest.mark.parametrize("lengths", [[512], [10, 129, 257, 1500], [1, 0, 1023], [511, 513, 515], [97, 1700], [130, 385]])
@pytest.mark.parametrize("D", [72, 128])
def test_windows_of_many_lengths(mp, D, lengths, window):
    c = Case(lengths, 2, 1, D, window=window, seed=len(lengths) + window)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()


@pytest.mark.parametrize("lengths", [[513], [1500], [129, 1, 31, 33, 65, 96], [1300, 97]])
@pytest.mark.parametrize("D", [72, 128])
def test_all_keys_of_many_lengths(mp, D, lengths):
    c = Case(lengths, 2, 2, D, causal=False, seed=D, before=3, after=5)
    c.forward(mp)
    c.check_forward()
    c.check_untouched()


@pytest.mark.parametrize("std,scale", [(8.0, 1.0), (0.01, 0.05), (30.0, 0.2)])
@pytest.mark.parametrize("D", [72, 128])
def test_sharp_and_flat_rows(mp, D, std, scale):
    c = Case([600], 2, 2, D, std=std, scale=scale)
    c.forward(mp)
    c.check_forward()
    c.backward(mp)
    c.check_backward()


@pytest.mark.parametrize("D,causal,window", [(64, True, 0), (64, True, 1000), (128, True, 0), (128, True, 1000), (128, False, 0)])
def test_long_sequences(mp, D, causal, window):
    c = Case([5000, 16384], 2, 1, D, causal, window)
    c.forward(mp)
    long = Case([16384], 2, 1, D, causal, window, before=5000)        # the same numbers, seen as one sequence
    for name in ("q", "k", "v", "o", "lse"):
        setattr(long, name, getattr(c, name))
    rows = torch.cat([torch.arange(0, 16384, 41, device="cuda"), torch.arange(16384 - 300, 16384, device="cuda")])
    for h in range(2):
        check_rows(long, rows, h)


@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 700)])
def test_backward_of_a_long_sequence(mp, D, window):
    c = Case([8192], 1, 1, D, window=window)
    c.forward(mp)
    c.backward(mp)
    c.check_backward()
