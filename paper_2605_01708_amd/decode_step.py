"""Continuous batching over a paged KV cache of 4-bit words, through the public calls of this package:

    python -m paper_2605_01708_amd.decode_step [--sequences 8] [--tokens 300] [--steps 12] [--layers 2]

Requests come with prompts of different lengths.  Each step asks for rows -- a prompt's, or one token --, cache_allot finds them pages
and writes the block table, lengths and starts that the other calls read; per layer, cache_append norms and rotates the projections
and writes K and V, and cache_attention reads what is there.  Requests that are done give their pages back and others take
their places; a step that the pool has too few pages for leaves everything as it is and is tried again without its newest request.  Values are
random: the weights of a model are not what is shown.  Steps of one token per sequence are captured into a graph once and replayed."""
from __future__ import annotations

import argparse

import torch

import paper_2605_01708_amd as sz

KV_HEADS, GROUP, DIM, PAGE = 8, 4, 128, 16


class Batch:
    """Buffers of a batch of up to n sequences of up to `most` tokens each, with a pool of `pages` pages in every layer."""

    def __init__(self, n: int, most: int, pages: int, layers: int, dtype: int = sz.FP4_E2M1, device: str = "cuda"):
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)   # noqa: E731
        self.n, self.most, self.device = n, most, device
        self.table, self.starts, self.lens, self.asked, self.kept = i32(n, -(-most // PAGE)), i32(n + 1), i32(n), i32(n), i32(n)
        self.pool = sz.PagePool.full(pages, PAGE, device)
        self.caches = [sz.KvCache.zeros(pages, PAGE, KV_HEADS, DIM, dtype, device) for _ in range(layers)]
        freqs = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
        weight = torch.ones(DIM, dtype=torch.bfloat16, device=device)
        self.how = sz.Rotation(freqs.float().to(device), eps=1e-6, q_weight=weight, k_weight=weight)
        self.attention = sz.Attention(DIM ** -0.5)

    def allot(self, rows, keep=None) -> dict:
        """A step's pages; rows and keep per sequence.  The pool's state."""
        self.asked.copy_(torch.tensor(rows, dtype=torch.int32))
        if keep is not None:
            self.kept.copy_(torch.tensor(keep, dtype=torch.int32))
        sz.cache_allot(self.pool, self.sequences(max(1, max(rows))), self.asked, keep=None if keep is None else self.kept)
        return sz.read_pool_state(self.pool)

    def sequences(self, max_rows: int) -> sz.Sequences:
        return sz.Sequences(self.table, self.starts, self.lens, max_rows, self.most)

    def layers(self, qkv, outs, max_rows: int) -> None:
        """qkv: per layer the projections [rows, q_heads + 2 kv_heads, dim]; outs: the attention's results.  The projections' Q is rotated in place."""
        seqs, heads = self.sequences(max_rows), KV_HEADS * GROUP
        for cache, x, out in zip(self.caches, qkv, outs):
            q, k, v = x[:, :heads], x[:, heads:heads + KV_HEADS], x[:, heads + KV_HEADS:]
            sz.cache_append(q, k, v, cache, seqs, self.how, q)
            sz.cache_attention(q, cache, seqs, out, sz.attention_workspace(cache, seqs, x.shape[0], heads, self.device), self.attention)


def serve(sequences: int = 8, tokens: int = 300, steps: int = 12, layers: int = 2, pages: int | None = None, device: str = "cuda"):
    """Admits prompts, decodes `steps` tokens with a captured step, ends every second request and admits as many again.  Returns the outputs of the last
    step per layer, the lengths, and how many requests had to wait for pages."""
    if sequences < 1 or tokens < sequences or steps < 1 or layers < 1:
        raise ValueError("there is a sequence, a step and a layer at least, and a token for each sequence")
    prompts = [tokens - tokens // sequences * s // 2 for s in range(sequences)]   # ragged
    most = tokens + 2 * steps
    batch = Batch(sequences, most, pages or sequences * -(-most // PAGE), layers, device=device)
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    heads = KV_HEADS * (GROUP + 2)
    waited = 0

    def values(n):
        return [torch.randn(n, heads, DIM, generator=gen, device=device).to(torch.bfloat16) for _ in range(layers)]

    def outputs(n):
        return [torch.empty(n, KV_HEADS * GROUP, DIM, dtype=torch.bfloat16, device=device) for _ in range(layers)]

    def admit(rows):
        """prompts of so many tokens each, the last of them left out as long as there are too few pages"""
        nonlocal waited
        while batch.allot(rows)["status"] & sz.ALLOT_PAGES:
            waited += 1
            rows = list(rows)
            rows[max(s for s, n in enumerate(rows) if n)] = 0
        if sum(rows):
            batch.layers(values(sum(rows)), outputs(sum(rows)), max(rows))
        return rows

    there = [n > 0 for n in admit(prompts)]
    # one token of each sequence: captured with its buffers, replayed with other values in them
    qkv, outs, one = values(sequences), outputs(sequences), batch.asked
    one.copy_(torch.tensor([int(x) for x in there], dtype=torch.int32))
    seqs, q_heads = batch.sequences(1), KV_HEADS * GROUP
    workspace = sz.attention_workspace(batch.caches[0], seqs, sequences, q_heads, device)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sz.cache_allot(batch.pool, seqs, one)
        for cache, x, out in zip(batch.caches, qkv, outs):
            sz.cache_append(x[:, :q_heads], x[:, q_heads:q_heads + KV_HEADS], x[:, q_heads + KV_HEADS:], cache, seqs, batch.how, x[:, :q_heads])
            sz.cache_attention(x[:, :q_heads], cache, seqs, out, workspace, batch.attention)
    for _ in range(steps):
        for x, y in zip(qkv, values(sequences)):
            x.copy_(y)
        graph.replay()

    # every second request ends, and another one takes its place
    lens = batch.lens.tolist()
    batch.allot([0] * sequences, keep=[0 if s % 2 else n for s, n in enumerate(lens)])
    again = admit([prompts[s] if s % 2 else 0 for s in range(sequences)])
    one.copy_(torch.tensor([int(there[s] if s % 2 == 0 else again[s] > 0) for s in range(sequences)], dtype=torch.int32))
    for x, y in zip(qkv, values(sequences)):
        x.copy_(y)
    graph.replay()
    return outs, batch.lens.tolist(), waited, batch


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("sequences", 8), ("tokens", 300), ("steps", 12), ("layers", 2)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--pages", type=int, default=None, help="of the pool (as many as all sequences need at most)")
    a = p.parse_args()
    try:
        outs, lens, waited, batch = serve(a.sequences, a.tokens, a.steps, a.layers, a.pages)
    except ValueError as e:
        p.error(str(e))
    torch.cuda.synchronize()
    print(f"{len(outs)} layers, sequences of {lens} tokens; {sz.read_pool_state(batch.pool)['free']} of {batch.pool.free.numel()} pages are free; "
          f"{waited} requests had to wait for pages")


if __name__ == "__main__":
    main()
