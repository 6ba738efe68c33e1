"""One decoding step with drafted tokens over a quantised, paged KV cache, and the cache's way to another node, through the public
calls of this package:

    python -m paper_2605_01708_amd.tree_decode [--tokens 2000] [--sequences 4] [--layers 4] [--drafts 13]

Per layer, a prompt is written into an E5M2 cache (cache_write), a tree of drafted tokens behind it, and all drafts attend to what they may see
(cache_attention); the longest path of the tree counts as accepted and becomes contiguous in all layers at once
(cache_move).  One sequence's pages of all layers then go through the codec (compress_batch_paged, decompress_batch_paged) into another
pool, their scales beside them, and are read back as BF16 there (cache_read).  Values are random: the weights of a model are not what is shown."""
from __future__ import annotations

import argparse

import torch

import paper_2605_01708_amd as sz

KV_HEADS, GROUP, DIM, PAGE = 8, 4, 128, 16


def tree_of(rows: int, branches: int = 3):
    """Bits of the ancestors (and itself) of every row, depths, and the path to the deepest row: row i hangs below (i - 1) // branches."""
    bits, depth = [1], [0]
    for i in range(1, rows):
        bits.append(bits[(i - 1) // branches] | 1 << i)
        depth.append(depth[(i - 1) // branches] + 1)
    path, at = [], rows - 1
    while at >= 0:
        path.append(at)
        at = (at - 1) // branches if at else -1
    return [b - (1 << 64) if b >> 63 else b for b in bits], depth, path[::-1]


def step(tokens: int = 2000, sequences: int = 4, layers: int = 4, drafts: int = 13, device: str = "cuda"):
    """Runs the step; returns the attention's outputs per layer, the accepted sequences' lengths, the codec's ratio and whether what arrived
    is what was sent."""
    if sequences < 1 or layers < 1 or not 1 <= drafts <= 64 or tokens <= 37 * (sequences - 1):
        raise ValueError("a step has a sequence and a layer at least, 1 to 64 drafts (the bits of a word), and more tokens than the 37 by which each "
                         "prompt is shorter than the one before it")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device)   # noqa: E731
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    prompts = [tokens - 37 * s for s in range(sequences)]               # ragged
    pages_of = [-(-(n + drafts) // PAGE) for n in prompts]
    pool = sum(pages_of)
    order = torch.randperm(pool, generator=gen, device=device).to(torch.int32)
    table = torch.zeros(sequences, max(pages_of), dtype=torch.int32, device=device)
    at = 0
    for s, n in enumerate(pages_of):
        table[s, :n] = order[at:at + n]
        at += n
    caches = [sz.KvCache.zeros(pool, PAGE, KV_HEADS, DIM, sz.FP8_E5M2, device) for _ in range(layers)]

    def rows(n, heads):
        return torch.randn(n, heads, DIM, generator=gen, device=device).to(torch.bfloat16)

    # the prompts, all rows of a call one behind the other
    starts = [sum(prompts[:s]) for s in range(sequences + 1)]
    prompt = sz.Sequences(table, i32(starts), i32(prompts), max_rows=max(prompts), max_len=max(prompts))
    for cache in caches:
        sz.cache_write(rows(starts[-1], KV_HEADS), rows(starts[-1], KV_HEADS), cache, prompt)

    # the drafts: written behind the prompt, then every one attends to the prompt and to its ancestors
    bits, depth, path = tree_of(drafts)
    n = drafts * sequences
    seqs = sz.Sequences(table, i32([drafts * s for s in range(sequences + 1)]), i32([p + drafts for p in prompts]), max_rows=drafts,
                        max_len=max(prompts) + drafts)
    how = sz.Attention(DIM ** -0.5, tree=torch.tensor(bits, device=device).repeat(sequences)[:, None].contiguous(),
                       positions=i32([p + d for p in prompts for d in depth]))
    workspace = sz.attention_workspace(caches[0], seqs, n, KV_HEADS * GROUP, device)
    outs = []
    for cache in caches:
        sz.cache_write(rows(n, KV_HEADS), rows(n, KV_HEADS), cache, seqs)
        q = rows(n, KV_HEADS * GROUP)
        out = torch.empty_like(q)
        sz.cache_attention(q, cache, seqs, out, workspace, how)
        outs.append(out)

    # the accepted path moves to the front of the drafts; a sequence is as long as its prompt and the path then
    sz.cache_move(sz.KvCaches(caches), seqs, i32([path] * sequences))
    lens = [p + len(path) for p in prompts]

    # sequence 0 goes to another node: the words of its whole pages through the codec, its scales as they are
    elems = pages_of[0] * PAGE * KV_HEADS * DIM
    mine = table[0, :pages_of[0]].contiguous()
    paging = sz.Paged(caches[0].k, mine, PAGE * KV_HEADS * DIM, PAGE * KV_HEADS * DIM)
    words = [t for cache in caches for t in (cache.k, cache.v)]
    sample = caches[0].k[mine[0].long()].cpu().reshape(-1)
    cb = sz.calibrate(sample, sz.FP8_E5M2)
    streams = [torch.empty(sz.compress_bound(elems, sz.FP8_E5M2), dtype=torch.uint8, device=device) for _ in words]
    sizes = sz.new_sizes_array(len(words), device)
    sz.CompressBatchPaged(words, [elems] * len(words), [cb] * len(words), streams, paging).launch(sz.Workspace(elems, sz.FP8_E5M2, device), sizes)
    sent = sz.read_sizes_array(sizes)
    there = [sz.KvCache.zeros(pages_of[0], PAGE, KV_HEADS, DIM, sz.FP8_E5M2, device) for _ in range(layers)]
    new_table = torch.arange(pages_of[0], dtype=torch.int32, device=device)
    new_paging = sz.Paged(there[0].k, new_table, PAGE * KV_HEADS * DIM, PAGE * KV_HEADS * DIM)
    sz.DecompressBatchPaged(streams, [s[0] for s in sent], [elems] * len(words), [cb] * len(words), [t for cache in there for t in (cache.k, cache.v)],
                            new_paging).launch()
    same = True
    for here, cache in zip(caches, there):
        cache.k_scales.copy_(here.k_scales[mine.long()])
        cache.v_scales.copy_(here.v_scales[mine.long()])
        got = [torch.empty(lens[0], KV_HEADS, DIM, dtype=torch.bfloat16, device=device) for _ in range(4)]
        sz.cache_read(here, sz.Sequences(mine[None].contiguous(), i32([0, lens[0]]), i32([lens[0]]), lens[0], lens[0]), *got[:2])
        sz.cache_read(cache, sz.Sequences(new_table[None].contiguous(), i32([0, lens[0]]), i32([lens[0]]), lens[0], lens[0]), *got[2:])
        same = same and torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])
    return outs, lens, elems * len(words) / sum(s[0] for s in sent), same


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=2000)
    p.add_argument("--sequences", type=int, default=4)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--drafts", type=int, default=13)
    a = p.parse_args()
    try:
        outs, lens, ratio, same = step(a.tokens, a.sequences, a.layers, a.drafts)
    except ValueError as e:
        p.error(str(e))
    torch.cuda.synchronize()
    print(f"{len(outs)} layers, outputs {tuple(outs[0].shape)}; sequences of {lens} tokens after the accepted path; "
          f"one of them sent at a ratio of {ratio:.3f}, {'as it was' if same else 'CHANGED'}")


if __name__ == "__main__":
    main()
