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
