"""Whatever tables, lengths, starts and paths say, the cache calls write into their buffers and nowhere else, and read what lies around these in no
call whose arguments are consistent.

Every buffer is a slice of a larger one, as many bytes as the call needs, between two stretches of a pattern."""
import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz

ROOM, PATTERN = 1 << 16, 0xa5


class Guarded:
    def __init__(self):
        self.all = []

    def __call__(self, *shape, dtype, fill=None):
        n = int(np.prod(shape)) * dtype.itemsize
        whole = torch.full((ROOM + n + (-n % 256) + ROOM,), PATTERN, dtype=torch.uint8, device="cuda")
        t = whole[ROOM:ROOM + n].view(dtype).view(shape)
        if fill is not None:
            t.copy_(torch.as_tensor(fill, device="cuda"))
        self.all.append((whole, n))
        return t

    def intact(self):
        torch.cuda.synchronize()
        return all(bool((w[:ROOM] == PATTERN).all()) and bool((w[ROOM + n:] == PATTERN).all()) for w, n in self.all)


def calls(kind, rows, group, tree, lens, starts, table, max_len, heads=2, dim=64, page=16, pages=5, n_rows=None, path=((0, 2, 7), (1, 0, -1))):
    """all four calls over two sequences; whether what lies around their buffers is as it was"""
    g = Guarded()
    word = torch.bfloat16 if kind == sz.BF16 else torch.uint8
    n = 2 * rows if n_rows is None else n_rows
    gen = torch.Generator("cuda")
    gen.manual_seed(rows)
    k, v = (g(pages, page, heads, dim, dtype=word, fill=torch.randint(0, 60, (pages, page, heads, dim), device="cuda", generator=gen).to(word)) for _ in range(2))
    scales = [None if kind == sz.BF16 else g(pages, heads, page, dtype=torch.uint8, fill=torch.full((pages, heads, page), 120)) for _ in range(2)]
    cache = sz.KvCache(k, v, kind, *scales)
    i32 = lambda *x: g(len(x), dtype=torch.int32, fill=torch.tensor(x, dtype=torch.int32))   # noqa: E731
    block_table = g(2, len(table[0]), dtype=torch.int32, fill=torch.tensor(table, dtype=torch.int32))
    seqs = sz.Sequences(block_table, i32(*starts), i32(*lens), rows, max_len)
    new = [g(n, heads, dim, dtype=torch.bfloat16, fill=torch.randn(n, heads, dim, device="cuda", generator=gen)) for _ in range(2)]
    back = [g(n, heads, dim, dtype=torch.bfloat16) for _ in range(2)]
    q, out = (g(n, heads * group, dim, dtype=torch.bfloat16, fill=torch.randn(n, heads * group, dim, device="cuda", generator=gen)) for _ in range(2))
    lse = g(n, heads * group, dtype=torch.float32)
    bits = g(n, 1, dtype=torch.int64, fill=torch.full((n, 1), 5)) if tree else None
    positions = g(n, dtype=torch.int32, fill=torch.arange(n, dtype=torch.int32) * 7) if tree else None
    sz.cache_write(new[0], new[1], cache, seqs)
    assert g.intact()
    sz.cache_read(cache, seqs, back[0], back[1])
    assert g.intact()
    for window in (0, 9):
        for softcap in (0.0, 20.0):
            how = sz.Attention(0.1, softcap=softcap, window=window, tree=bits, positions=positions)
            workspace = g(sz.attention_workspace_bytes(cache, seqs, n, heads * group), dtype=torch.uint8)
            sz.cache_attention(q, cache, seqs, out, workspace, how, lse)
            assert g.intact()
    sz.cache_move(sz.KvCaches([cache]), seqs, g(2, 3, dtype=torch.int32, fill=torch.tensor(path, dtype=torch.int32)), n_rows=n)
    assert g.intact()
    return out


KINDS = [sz.BF16, sz.FP8_E5M2, sz.FP8_E4M3]
GOOD = [[0, 3, 1], [2, 4, 4]]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,group", [(2, 1), (3, 4), (6, 3), (20, 2), (9, 8)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("max_len", [48, 9000])
def test_consistent_arguments(kind, rows, group, tree, max_len):
    """up to 16 rows and more, whole sequences and parts of them"""
    out = calls(kind, rows, group, tree, [40, rows], [0, rows, 2 * rows], GOOD, max_len)
    assert torch.isfinite(out.float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,group", [(2, 1), (6, 3)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("max_len", [48, 9000])
@pytest.mark.parametrize("lens,starts,table", [([1 << 30, -5], None, GOOD), ([(1 << 31) - 1, -(1 << 31)], None, GOOD), ([40, 48], [-3, 2, 1 << 20], GOOD),
                                               ([40, 48], [3, 1, 4], GOOD), ([40, 48], [(1 << 31) - 1, -(1 << 31), (1 << 31) - 1], GOOD),
                                               ([40, 48], None, [[-1] * 3] * 2), ([40, 48], None, [[5, 1 << 30, 0], [0, 6, 99]]), ([1, 2], None, GOOD)])
def test_arguments_that_say_anything(kind, rows, group, tree, max_len, lens, starts, table):
    """lengths, starts and page indices beyond the buffers, or shorter than the rows"""
    calls(kind, rows, group, tree, lens, [0, rows, 2 * rows] if starts is None else starts, table, max_len)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("path", [((1 << 30, 0, 0), (-5, 1, 2)), ((0, 5, (1 << 31) - 1), (2, 2, 2)), ((-(1 << 31), 0, 1), (5, 4, 3))])
def test_paths_that_say_anything(kind, path):
    calls(kind, 6, 1, True, [40, 48], [0, 6, 12], GOOD, 48, path=path)
