"""What an FP8 cache makes of the largest values: where a word stands for 2^128, it is read as an infinity and attended to as one."""
import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("kind,least,below", [(sz.FP8_E5M2, 1.875, 1.75), (sz.FP8_E4M3, 1.9375, 1.875)])
def test_the_largest_finite_values(kind, least, below, T):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    x = torch.ones(2, T, 1, 64)
    edge = float(np.float32(least) * np.float32(2.0) ** 127)
    x[1, 0, 0, 3] = edge                                                                   # of V alone: the scores stay numbers
    x[1, 0, 0, 4] = -edge
    before = torch.tensor(edge).to(torch.bfloat16).view(torch.int16) - 1                   # the BF16 number in front of it
    x[1, 0, 0, 5] = before.view(torch.bfloat16).float()
    x = x.to(torch.bfloat16).cuda()
    cache = sz.KvCache.zeros(1, 64, 1, 64, kind)
    seqs = sz.Sequences(None, i32(0, T), i32(T), T, T)
    sz.cache_write(x[0], x[1], cache, seqs)
    y = torch.zeros_like(x)
    sz.cache_read(cache, seqs, y[0], y[1])
    row = y[1, 0, 0].double().cpu()
    assert row[3] == float("inf") and row[4] == -float("inf") and row[5] == below * 2.0 ** 127
    q = torch.ones(T, 1, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    sz.cache_attention(q, cache, seqs, out, sz.attention_workspace(cache, seqs, T, 1), sz.Attention(0.1))
    out = out[:, 0].double().cpu()
    assert torch.isposinf(out[:, 3]).all() and torch.isneginf(out[:, 4]).all() and torch.isfinite(out[:, [k for k in range(64) if k not in (3, 4)]]).all()
