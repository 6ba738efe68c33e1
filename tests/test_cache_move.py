"""splitzip_cache_move over geometries and lengths of paths: every word and every scale is where the path puts it, and nothing else has moved."""
import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz

KINDS = [sz.BF16, sz.FP8_E5M2, sz.FP8_E4M3]


def moved(kind, heads, dim, lengths, rows, page=16, layers=2, seed=0):
    """One call over sequences whose paths have these lengths (of `rows` drafted tokens each): what it left, and what it should have."""
    rng = np.random.default_rng(seed)
    lens = [rows + int(x) for x in rng.integers(0, 3 * page, len(lengths))]
    width = -(-max(lens) // page)
    pages = len(lens) * width + 1
    table = rng.permutation(pages)[:-1].reshape(len(lens), width).astype(np.int32)
    paths = np.full((len(lens), max(lengths)), -1, np.int32)
    for s, n in enumerate(lengths):
        paths[s, :n] = np.sort(rng.choice(rows, n, replace=False))
    es, word = (2, torch.int16) if kind == sz.BF16 else (1, torch.uint8)
    gen = torch.Generator()
    gen.manual_seed(seed)
    words = torch.randint(0, 256, (layers, 2, pages, page, heads, dim * es), generator=gen, dtype=torch.uint8).view(word)
    scales = torch.randint(0, 255, (layers, 2, pages, heads, page), generator=gen, dtype=torch.uint8)
    on = words.cuda(), scales.cuda()
    caches = [sz.KvCache(w[0], w[1], kind, *([None, None] if kind == sz.BF16 else b)) for w, b in zip(*on)]
    starts = torch.arange(len(lens) + 1, dtype=torch.int32) * rows
    seqs = sz.Sequences(torch.from_numpy(table).cuda(), starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), rows, max(lens))
    sz.cache_move(sz.KvCaches(caches), seqs, torch.from_numpy(paths).cuda())
    want = words.clone(), scales.clone()
    for s, n in enumerate(lengths):
        at = lens[s] - rows + np.arange(n)
        frm = lens[s] - rows + paths[s, :n]
        (p0, t0), (p1, t1) = (table[s, frm // page], frm % page), (table[s, at // page], at % page)
        want[0][:, :, p1, t1] = words[:, :, p0, t0]
        if kind != sz.BF16:
            want[1].transpose(3, 4)[:, :, p1, t1] = scales.transpose(3, 4)[:, :, p0, t0]
    return [t.cpu() for t in on], want


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [1, 2, 4, 5, 7, 8, 13])
def test_every_entry_of_a_path_moves(kind, heads, dim):
    """pieces of a token that leave the last wave of a workgroup any number of lanes, under paths of more entries than these"""
    got, want = moved(kind, heads, dim, [1, 3, 4, 5, 6, 7, 9, 17, 20, 33, 40, 63, 64], 70, seed=heads + dim)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,dim", [(1, 64), (2, 256), (4, 128), (3, 64)])
def test_paths_of_more_than_64_entries_move(kind, heads, dim):
    got, want = moved(kind, heads, dim, [65, 70, 64, 128, 129, 130, 200, 2], 200, seed=3)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
