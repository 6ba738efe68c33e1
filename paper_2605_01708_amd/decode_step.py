"""Continuous batching over a paged KV cache of 4-bit words, through the public calls of this package:

    python -m paper_2605_01708_amd.decode_step [--sequences 8] [--tokens 300] [--steps 12] [--layers 2] [--pages N]

Requests come with prompts of different lengths.  Each step asks for rows -- a prompt's, or one token --, cache_allot finds them pages
and writes the block table, lengths and starts that the other calls read; per layer, cache_append norms and rotates the projections
and writes K and V, and cache_attention reads what is there.  Requests that are done give their pages back and others take
their places.  A step that the pool has too few pages for leaves everything as it is: prompts are asked for again without the last of them; of the
requests that decode, the newest gives its pages back and waits until there are enough for all of its tokens, and the others' step is taken
again with the same projections.  Values are random: the weights of a model are not what is shown.  Steps of one token per sequence are captured
into a graph once and replayed; what became of a step is read after each."""
from __future__ import annotations

import argparse

import torch

import paper_2605_01708_amd as sz

KV_HEADS, GROUP, DIM, PAGE = 8, 4, 128, 16
ALL = 1 << 30   # tokens that a sequence keeps: more than it can have


def _pages(tokens: int) -> int:
    return -(-tokens // PAGE)


class Batch:
    """Buffers of a batch of up to n sequences of up to `most` tokens each, with a pool of `pages` pages in every layer."""

    def __init__(self, n: int, most: int, pages: int, layers: int, dtype: int = sz.FP4_E2M1, device: str = "cuda"):
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)   # noqa: E731
        self.n, self.most, self.device = n, most, device
        self.table, self.starts, self.lens, self.asked, self.kept = i32(n, _pages(most)), i32(n + 1), i32(n), i32(n), i32(n)
        self.pool = sz.PagePool.full(pages, PAGE, device)
        self.caches = [sz.KvCache.zeros(pages, PAGE, KV_HEADS, DIM, dtype, device) for _ in range(layers)]
        freqs = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
        weight = torch.ones(DIM, dtype=torch.bfloat16, device=device)
        self.how = sz.Rotation(freqs.float().to(device), eps=1e-6, q_weight=weight, k_weight=weight)
        self.attention = sz.Attention(DIM ** -0.5)

    def ask(self, rows, keep=None) -> None:
        """What the next step is to have: rows, and the tokens that are kept (None: all), per sequence."""
        self.asked.copy_(torch.tensor(rows, dtype=torch.int32))
        self.kept.copy_(torch.tensor([ALL] * self.n if keep is None else keep, dtype=torch.int32))

    def allot(self, rows, keep=None) -> dict:
        """A step's pages; rows and keep per sequence.  The pool's state."""
        self.ask(rows, keep)
        sz.cache_allot(self.pool, self.sequences(max(1, max(rows))), self.asked, keep=self.kept)
        return self.state()

    def state(self) -> dict:
        """What became of the last step: taken (status 0), or left for too few pages."""
        state = sz.read_pool_state(self.pool)
        if state["status"] & ~sz.ALLOT_PAGES:
            raise RuntimeError(f"a step that no number of pages helps: {state}")
        return state

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
    """Admits prompts, decodes `steps` tokens with a captured step, ends every second request, admits as many again and decodes one more.  Returns
    the outputs of the last step per layer (a row for each sequence that it had, batch.running), the lengths, how often a request had to wait for pages,
    and the batch.  batch.queries: what those rows asked with; batch.prompts and batch.decoded: the tokens of each sequence's request."""
    if sequences < 1 or tokens < sequences or steps < 1 or layers < 1:
        raise ValueError("there is a sequence, a step and a layer at least, and a token for each sequence")
    prompts = [tokens - tokens // sequences * s // 2 for s in range(sequences)]   # ragged
    most = tokens + 2 * steps
    if pages is None:
        pages = sequences * _pages(most)
    if pages < _pages(tokens + steps + 1):   # (then the oldest request can always go on)
        raise ValueError(f"the longest request, of {tokens + steps + 1} tokens at its end, needs {_pages(tokens + steps + 1)} pages")
    batch = Batch(sequences, most, pages, layers, device=device)
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    heads = KV_HEADS * (GROUP + 2)
    running, waiting, decoded, waited = [], list(range(sequences)), [0] * sequences, 0   # running: in the order in which they came

    def values(n):
        return [torch.randn(n, heads, DIM, generator=gen, device=device).to(torch.bfloat16) for _ in range(layers)]

    def outputs(n):
        return [torch.zeros(n, KV_HEADS * GROUP, DIM, dtype=torch.bfloat16, device=device) for _ in range(layers)]

    def admit(ready):
        """the waiting requests of these sequences, with all tokens that they have so far; the last of them left out as long as there are too few pages"""
        nonlocal waited
        ready = list(ready)
        while ready:
            rows = [prompts[s] + decoded[s] if s in ready else 0 for s in range(sequences)]
            if not batch.allot(rows)["status"]:
                batch.layers(values(sum(rows)), outputs(sum(rows)), max(rows))
                break
            waited += 1
            ready.pop()
        for s in ready:
            waiting.remove(s)
            running.append(s)

    def admit_what_fits(state):
        """of those that wait, as many as there are pages for, and for the next token of all"""
        free, ready = state["free"] - sum((prompts[s] + decoded[s]) % PAGE == 0 for s in running), []
        for s in waiting:
            free -= _pages(prompts[s] + decoded[s] + 1)
            if free < 0:
                break
            ready.append(s)
        admit(ready)

    admit(waiting)
    # one token of each sequence: captured with its buffers, replayed with other values in them
    qkv, outs = values(sequences), outputs(sequences)
    seqs, q_heads = batch.sequences(1), KV_HEADS * GROUP
    workspace = sz.attention_workspace(batch.caches[0], seqs, sequences, q_heads, device)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sz.cache_allot(batch.pool, seqs, batch.asked, keep=batch.kept)
        for cache, x, out in zip(batch.caches, qkv, outs):
            sz.cache_append(x[:, :q_heads], x[:, q_heads:q_heads + KV_HEADS], x[:, q_heads + KV_HEADS:], cache, seqs, batch.how, x[:, :q_heads])
            sz.cache_attention(x[:, :q_heads], cache, seqs, out, workspace, batch.attention)

    def decode():
        """a token of every request that runs, the rows in the sequences' order"""
        nonlocal waited
        keep = [ALL] * sequences
        for x, y in zip(qkv, values(len(running))):
            x[:len(running)] = y
        while True:
            batch.ask([int(s in running) for s in range(sequences)], keep)
            graph.replay()
            state = batch.state()
            if not state["status"]:
                break
            newest = running.pop()   # gives its pages back; nothing of the step has been done, its row goes out of the projections
            row = sum(s < newest for s in running)
            for x in qkv:
                x[row:len(running)] = x[row + 1:len(running) + 1].clone()
            keep[newest] = 0
            waiting.insert(0, newest)
            waited += 1
        for s in running:
            decoded[s] += 1
        return state

    for _ in range(steps):
        admit_what_fits(decode())

    # every second request ends, and another one takes its place behind those that wait
    ended = [s for s in running if s % 2]
    state = batch.allot([0] * sequences, keep=[0 if s in ended else ALL for s in range(sequences)])
    for s in ended:
        running.remove(s)
        decoded[s] = 0
    waiting += ended
    admit_what_fits(state)
    waited += sum(s in waiting for s in ended)
    decode()
    n = len(running)
    batch.running, batch.prompts, batch.decoded, batch.queries = sorted(running), prompts, decoded, [x[:n, :q_heads] for x in qkv]
    return [o[:n] for o in outs], batch.lens.tolist(), waited, batch


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
          f"a request had to wait for pages {waited} times")


if __name__ == "__main__":
    main()
