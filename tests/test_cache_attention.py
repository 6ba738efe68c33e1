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


@pytest.mark.gpu
@pytest.mark.parametrize("n,T", [(1, 1), (1, 200), (2, 70), (3, 9), (5, 33), (16, 17), (33, 3), (64, 2), (70, 1), (130, 4)])
@pytest.mark.parametrize("hint", [None, 5000])
def test_positions_under_a_window(n, T, hint):
    """the row at the lowest position, wherever it is among a sequence's rows and whatever number of lanes looks for it, decides where the
    sequence begins; some sequences have no rows, more than 64 are counted in turns, and a hint of long ones cuts short ones into parts"""
    rng = np.random.default_rng(n + T)
    rows = [T if k % 4 != 3 else int(rng.integers(0, T + 1)) for k in range(n)]
    lens = [r + int(rng.integers(0, 300 if n < 64 else 200)) for r in rows]
    w = World(sz.FP8_E4M3 if n % 2 else sz.BF16, lens, rows, 1, 64, 16, seed=n, max_len=hint)
    pos = np.concatenate([[max(0, L - r) + rng.permutation(r)] for L, r in zip(lens, rows)], axis=None).astype(np.int64)
    for s in range(n):   # one row far in front of the others
        if rows[s] > 2:
            pos[w.starts[s] + int(rng.integers(rows[s]))] -= 60
    q, qd = queries(w, 2)
    how = sz.Attention(0.1, window=40, positions=torch.from_numpy(pos.astype(np.int32)).cuda())
    close(*run(w, qd, how), attend(w, q, 0.1, window=40, positions=pos))


@pytest.mark.gpu
def test_positions_of_a_prompt_do_not_wait_for_one_another():
    """a piece of a prompt of 2048 rows with positions and a window takes less than two and a half times what it takes without (four times
    if the positions were looked at one by one)"""
    T = 2048
    cache = sz.KvCache.zeros(T // 16, 16, 8, 128, sz.BF16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    seqs = sz.Sequences(torch.arange(T // 16, dtype=torch.int32, device="cuda")[None], i32(0, T), i32(T), T, T)
    q = torch.randn(T, 32, 128, device="cuda").to(torch.bfloat16)
    out, workspace = torch.empty_like(q), sz.attention_workspace(cache, seqs, T, 32)
    hows = [sz.Attention(0.1), sz.Attention(0.1, window=1 << 20, positions=torch.arange(T, dtype=torch.int32, device="cuda"))]
    took = [[], []]
    for k in range(20):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(5):
            sz.cache_attention(q, cache, seqs, out, workspace, hows[k % 2])
        b.record()
        torch.cuda.synchronize()
        took[k % 2].append(a.elapsed_time(b))
    assert min(took[1]) < 2.5 * min(took[0]), took


@pytest.mark.gpu
def test_an_infinity_is_looked_for_in_its_own_rows_alone():
    """one infinity of V in the first of the sequences that a workgroup takes costs what it does in the last one (seven times that, if
    the sequences behind it were searched as well), and touches no other sequence"""
    n, T = 4096, 200
    cache = sz.KvCache.zeros(n * 25, 8, 1, 64, sz.BF16)
    table = torch.arange(n * 25, dtype=torch.int32, device="cuda").view(n, 25)
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * T
    seqs = sz.Sequences(table, starts, torch.full((n,), T, dtype=torch.int32, device="cuda"), T, T)
    x = torch.randn(3, n * T, 1, 64, device="cuda").to(torch.bfloat16)
    sz.cache_write(x[0], x[1], cache, seqs)
    out, workspace, how = torch.empty_like(x[2]), sz.attention_workspace(cache, seqs, n * T, 1), sz.Attention(0.1)
    took, outs = [[], []], []
    for k in range(12):
        odd = (0, n - 1)[k % 2]
        was = cache.v[odd * 25, 3, 0, 5].clone()
        cache.v[odd * 25, 3, 0, 5] = float("inf")
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(5):
            sz.cache_attention(x[2], cache, seqs, out, workspace, how)
        b.record()
        torch.cuda.synchronize()
        took[k % 2].append(a.elapsed_time(b))
        outs.append(out.clone())
        cache.v[odd * 25, 3, 0, 5] = was
    first, last = outs[-2].view(n, T, 64), outs[-1].view(n, T, 64)
    assert torch.isposinf(first[0, 3:, 5]).all() and torch.isfinite(first[1:]).all() and torch.isfinite(first[0, :3]).all()
    assert torch.isposinf(last[-1, 3:, 5]).all() and torch.isfinite(last[:-1]).all()
    assert torch.equal(first[1:-1], last[1:-1])
    assert min(took[0]) < 2 * min(took[1]), took


def exactly(got, got_lse, want, tokens):
    """as `close`, with weights that are 2^-15 of themselves off at most in place of 2^-8, and sums over so many tokens in 32 bits"""
    out, lse, mean, dx = want
    got = got.double().cpu().numpy()
    bound = 2.0 ** -8 * 1.01 * np.abs(out) + (2.0 ** -15 * 1.01 + 2.5 * dx[..., None] + 2.0 ** -20 + 2.0 ** -23 * tokens[:, None, None]) * mean
    worst = np.abs(got - out) - bound
    assert (worst <= 0).all(), (worst.max(), (worst > 0).mean())
    assert (np.abs(got_lse.double().cpu().numpy() - lse) <= dx + 2.0 ** -20 * (1 + np.abs(lse))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [sz.BF16, sz.FP8_E5M2, sz.FP8_E4M3])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,T", [(1, 1), (4, 4), (16, 1)])
def test_weights_of_few_rows_keep_their_bits(kind, dim, group, T):
    """up to 16 rows of a head of the cache: the result's own rounding to BF16 is the only one that shows; whole sequences, and parts"""
    w = World(kind, [T + 30, T + 61, T + 900], [T] * 3, 1, dim, 16, seed=dim + T, max_len=9000)
    q, qd = queries(w, group)
    exactly(*run(w, qd, sz.Attention(0.01)), attend(w, q, 0.01), np.repeat(w.lens, w.rows))
