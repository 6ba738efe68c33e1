"""splitzip_cache_attention at the edges of its arguments: positions, windows, values and lengths where a form of a kernel ends."""
import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz
from test_cache_ops import World, attend, close, queries, run


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 40])
def test_positions_at_both_ends_of_their_range(T):
    """rows 2^31 apart: the bias of the one for the other keeps its sign"""
    w = World(sz.BF16, [60 + T, T], [T, T], 1, 64, 16, seed=21)
    q, qd = queries(w, 2)
    pos = [(-1 if i % 2 == 0 else 1) << 30 for i in range(T)] * 2
    slopes = np.array([2.0 ** -30, 2.0 ** -31])
    how = sz.Attention(0.1, slopes=torch.tensor(slopes, dtype=torch.float32, device="cuda"), positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    close(*run(w, qd, how), attend(w, q, 0.1, slopes=slopes, positions=pos))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("window", [1 << 31, (1 << 32) - 1, -1])
def test_a_window_wider_than_any_sequence_is_none(T, window):
    """the same bits as without a window, by the same way through the tokens: an infinity of V under a weight that is no number above 0
    shows which of the two a stage took"""
    w = World(sz.BF16, [300 + T, 2000 + T], [T, T], 1, 128, 16, seed=22)
    q, qd = queries(w, 2)
    qd[:] = 1.0
    w.set(0, 70, 0, 0, np.full(128, -64.0))
    w.set(0, 70, 1, 0, np.where(np.arange(128) == 9, np.inf, 1.0))
    out, lse = run(w, qd, sz.Attention(0.5))
    assert not torch.isfinite(out[:T, :, 9]).any() and torch.isfinite(out[T:]).all()
    again, lse2 = run(w, qd, sz.Attention(0.5, window=window))
    assert torch.equal(torch.isnan(out), torch.isnan(again)) and torch.equal(out.nan_to_num(), again.nan_to_num()) and torch.equal(lse, lse2)
