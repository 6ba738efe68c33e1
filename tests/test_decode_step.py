"""The operators of a step as a program runs them together: pages allotted, projections appended, attention over 4-bit words, captured and replayed
(paper_2605_01708_amd.decode_step), and the same against the formulas in 64 bits.

Attention's tolerance is that of the cache's own tests, over the values that the cache holds, whose words are checked where they are written."""
import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz
from test_cache_ops import attend, close

I32 = torch.int32


@pytest.mark.parametrize("args", [dict(sequences=0), dict(tokens=3, sequences=4), dict(steps=0), dict(layers=0)])
def test_the_example_says_what_it_takes(args):
    from paper_2605_01708_amd import decode_step

    with pytest.raises(ValueError, match="at least"):
        decode_step.serve(**args)


@pytest.mark.gpu
@pytest.mark.parametrize("args,waits", [(dict(sequences=8, tokens=300, steps=5, layers=2), False), (dict(sequences=1, tokens=1, steps=1, layers=1), False),
                                        (dict(sequences=5, tokens=200, steps=20, layers=1, pages=48), True)])
def test_the_example_runs(args, waits):
    from paper_2605_01708_amd import decode_step

    outs, lens, waited, batch = decode_step.serve(**args)
    torch.cuda.synchronize()
    assert (waited > 0) == waits and all(torch.isfinite(o).all() or waits for o in outs)
    state = sz.read_pool_state(batch.pool)
    used = [int(p) for s, n in enumerate(lens) for p in batch.table[s, :-(-n // decode_step.PAGE)].tolist()]
    free = batch.pool.free[:state["free"]].tolist()
    assert sorted(used + free) == list(range(batch.pool.free.numel()))          # every page is one sequence's, or free


class Held:
    """what a batch's cache holds, for the formulas"""

    def __init__(self, cache, table, lens, rows, dim, page):
        self.heads, self.dim, self.lens, self.rows = cache.kv_heads, dim, lens, rows
        self.starts = np.concatenate([[0], np.cumsum(rows)])
        self.table, self.page = table.cpu().numpy(), page
        value = []
        for words, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
            w = words.cpu()
            nibble = torch.stack([w & 15, w >> 4], -1).flatten(-2).numpy()
            x = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6])[nibble]
            value.append(x * np.repeat(np.exp2(scales.cpu().movedim(-1, 1).numpy() - 127.0), 32, -1))
        self.value = np.stack(value)

    def tokens(self, s, n):
        at = np.arange(n)
        return self.value[:, self.table[s, at // self.page], at % self.page]


@pytest.mark.gpu
@pytest.mark.parametrize("graph", [False, True])
def test_steps_against_the_formulas(graph):
    """prompts, then steps of one token, drafts that are given back, and a request that ends: what every step's attention sees is what was appended"""
    n, heads, group, dim, page, most = 4, 2, 3, 128, 16, 200
    gen = torch.Generator("cuda").manual_seed(1)
    i32 = lambda *s: torch.zeros(*s, dtype=I32, device="cuda")   # noqa: E731
    table, starts, lens, asked, keep = i32(n, -(-most // page)), i32(n + 1), i32(n), i32(n), i32(n)
    pool, cache = sz.PagePool.full(40, page), sz.KvCache.zeros(40, page, heads, dim, sz.FP4_E2M1)
    freqs = torch.rand(dim // 2, device="cuda")
    how, attention = sz.Rotation(freqs, eps=1e-6), sz.Attention(0.09)
    host = [0] * n
    plan = [([130, 1, 0, 60], None), ([1, 1, 1, 1], None), ([5, 5, 5, 5], None), ([1, 1, 1, 1], [131, 3, 1, 62]), ([0, 1, 17, 1], [0, 4, 2, 63]), ([33, 1, 1, 1], None)]
    for k, (rows, kept) in enumerate(plan):
        total = sum(rows)
        asked.copy_(torch.tensor(rows, dtype=I32))
        keep.copy_(torch.tensor([1 << 20] * n if kept is None else kept, dtype=I32))
        seqs = sz.Sequences(table, starts, lens, max(rows), most)
        x = torch.randn(total, heads * (group + 2), dim, generator=gen, device="cuda").to(torch.bfloat16)
        q, new_k, new_v = x[:, :heads * group], x[:, heads * group:heads * (group + 1)], x[:, heads * (group + 1):]
        positions, slots, of = i32(total + 3), torch.zeros(total + 3, dtype=torch.int64, device="cuda"), i32(total + 3)
        q_out, k_out, out = torch.empty_like(q), torch.empty_like(new_k), torch.empty(total, heads * group, dim, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(total, heads * group, device="cuda")
        ws = sz.attention_workspace(cache, seqs, total, heads * group)

        def step():
            sz.cache_allot(pool, seqs, asked, keep=keep, slots=slots, row_seqs=of, positions=positions)
            sz.cache_append(q, new_k, new_v, cache, seqs, how, q_out, k_out)
            sz.cache_attention(q_out, cache, seqs, out, ws, attention, lse)

        if graph and k:                                        # captured in a state that the replay then starts from
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step()
            captured.replay()
        else:
            step()
        torch.cuda.synchronize()
        host = [min(h, 1 << 20 if kept is None else kept[s]) + rows[s] for s, h in enumerate(host)]
        assert lens.tolist() == host and sz.read_pool_state(pool)["status"] == 0 and slots[total:].eq(-1).all()
        at = [host[s] - r + i for s, r in enumerate(rows) for i in range(r)]
        assert positions[:total].tolist() == at and of[:total].tolist() == [s for s, r in enumerate(rows) for _ in range(r)]
        # the rows' K stands where the slots say: within half of the words' widest step of what was appended
        held = Held(cache, table, host, rows, dim, page)
        flat = held.value.reshape(2, -1, heads, dim)[:, slots[:total].cpu().numpy()]
        for which, rounded in ((0, k_out), (1, new_v)):
            want = rounded.double().cpu().numpy()
            top = np.repeat(np.abs(want).reshape(total, heads, -1, 32).max(-1), 32, -1)
            assert (np.abs(flat[which] - want) <= top / 3 * 1.01).all()           # (a step is 2 of 6 at the top, and the power up to twice what it need be)
        close(out, lse, attend(held, q_out.double().cpu().numpy(), 0.09))


@pytest.mark.parametrize("pages", [-1, 0, 1])
def test_a_pool_that_no_request_fits_is_refused(pages):
    """16 tokens, one more by the captured step and one behind it: two pages"""
    from paper_2605_01708_amd import decode_step

    with pytest.raises(ValueError, match="needs 2 pages"):
        decode_step.serve(sequences=1, tokens=16, steps=1, layers=1, pages=pages)


@pytest.mark.gpu
@pytest.mark.parametrize("args,dry", [(dict(sequences=8, tokens=300, steps=5, layers=2), False), (dict(sequences=1, tokens=16, steps=1, layers=1, pages=2), False),
                                      (dict(sequences=5, tokens=200, steps=20, layers=1, pages=48), True), (dict(sequences=4, tokens=64, steps=40, layers=2, pages=16), True),
                                      (dict(sequences=6, tokens=90, steps=33, layers=1, pages=8), True)])
def test_no_step_is_lost_when_pages_run_out(args, dry):
    """the oldest request has a token of every step, a request its prompt and a token of each step that it was in, one that waits nothing; what the last step
    returns is attention over what the cache holds"""
    from paper_2605_01708_amd import decode_step

    outs, lens, waited, batch = decode_step.serve(**args)
    torch.cuda.synchronize()
    assert (waited > 0) == dry
    assert lens[0] == args["tokens"] + args["steps"] + 1
    if not dry:
        assert lens == [n + (1 if s % 2 else args["steps"] + 1) for s, n in enumerate(batch.prompts)]
    assert lens == [batch.prompts[s] + batch.decoded[s] if s in batch.running else 0 for s in range(batch.n)]
    rows = [int(s in batch.running) for s in range(batch.n)]
    for cache, q, out in zip(batch.caches, batch.queries, outs):
        held = Held(cache, batch.table, lens, rows, decode_step.DIM, decode_step.PAGE)
        assert out.shape == q.shape == (sum(rows), decode_step.KV_HEADS * decode_step.GROUP, decode_step.DIM)
        want, lse, mean, dx = attend(held, q.double().cpu().numpy(), decode_step.DIM ** -0.5)
        close(out, torch.from_numpy(lse), (want, lse, mean, dx))                    # (the program does not ask for lse)
