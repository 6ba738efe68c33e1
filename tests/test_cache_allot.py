"""Pages for a step's rows (splitzip_cache_allot) against the same on the host, one request and one page at a time.  All of it is whole numbers: exact."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz
from paper_2605_01708_amd.binding import _CPool, _CSeqs
from test_cache_guards import Guarded

I32, I64 = torch.int32, torch.int64


class Host:
    """the same buffers here"""

    def __init__(self, n, width, page, pages, free=None, lens=None, seed=0):
        self.page, self.width = page, width
        self.stack = np.random.default_rng(seed).permutation(pages).astype(np.int32)
        self.state = np.zeros(8, np.int32)
        self.state[0] = pages if free is None else free
        self.table, self.lens, self.starts = np.full((n, width), -7, np.int32), np.zeros(n, np.int32), np.zeros(n + 1, np.int32)

    def step(self, rows, keep=None, n_rows=1 << 30):
        """slots, sequences and positions of the step's rows, or None where it cannot be taken"""
        rows = np.maximum(rows, 0).astype(np.int64)
        room = min(self.width * self.page, 1 << 30)
        old = np.clip(self.lens.astype(np.int64), 0, room)
        kept = old if keep is None else np.minimum(np.maximum(keep, 0), old)
        new = kept + rows
        held, need = -(-old // self.page), -(-new // self.page)
        given, taken, free = int(np.maximum(held - need, 0).sum()), int(np.maximum(need - held, 0).sum()), int(self.state[0])
        status = (4 if (new > room).any() else 0) | (2 if rows.sum() > n_rows else 0)
        if free < 0 or free + given > len(self.stack):
            status |= 8
        elif taken > free + given:
            status |= 1
        self.starts[:] = 0
        self.state[1:] = [status, taken - free - given if status & 1 else 0, 0, 0, 0, 0, 0]
        if status:
            return None
        back = [self.table[s, p] for s in range(len(rows)) for p in range(need[s], held[s])]
        for r, p in enumerate(reversed(back)):
            self.stack[free + r] = p
        free += given
        out = [], [], []
        for s in range(len(rows)):
            for p in range(held[s], need[s]):
                free -= 1
                self.table[s, p] = self.stack[free]
            for t in range(kept[s], new[s]):
                for x, y in zip(out, (int(self.table[s, t // self.page]) * self.page + t % self.page, s, t)):
                    x.append(y)
        self.lens[:] = new
        self.starts[1:] = np.cumsum(rows)
        self.state[:] = [free, 0, 0, rows.sum(), rows.max(), new.max(), taken, given]
        return out


class Device:
    def __init__(self, h, make=None):
        t = lambda x: torch.from_numpy(x.copy()).cuda() if make is None else make(*x.shape, dtype=I32, fill=torch.from_numpy(x.copy()))   # noqa: E731
        self.table, self.lens, self.starts, self.free, self.state = t(h.table), t(h.lens), t(h.starts), t(h.stack), t(h.state)
        self.seqs, self.pool = sz.Sequences(self.table, self.starts, self.lens, 1, 1), sz.PagePool(self.free, self.state, h.page)

    def same(self, h):
        for a, b in ((self.table, h.table), (self.lens, h.lens), (self.starts, h.starts), (self.state, h.state), (self.free, h.stack)):
            assert np.array_equal(a.cpu().numpy(), b), (a, b)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=I32, device="cuda")


def outputs(n, make=None):
    make = make or (lambda *s, dtype: torch.full(s, 77, dtype=dtype, device="cuda"))
    return make(n, dtype=I64), make(n, dtype=I32), make(n, dtype=I32)


def compare(got, want, n):
    for t, x in zip(got, want or ([], [], [])):
        assert np.array_equal(t.cpu().numpy(), np.concatenate([np.array(x, np.int64), np.full(n - len(x), -1)]))


# ---- what is refused -----------------------------------------------------------------------------------

def test_descriptions_are_checked():
    L, buf = sz.lib(), 1 << 16

    def call(pool=None, seqs=None, rows=buf, keep=None, slots=None, of=None, pos=None, n=16):
        p = dict(free=buf, state=buf, pages=4, page=16, res=0)
        p.update(pool or {})
        q = dict(table=buf, starts=buf, lens=buf, stride=4, n=1 << 16, rows=1, len=64)          # (too many sequences: nothing is ever launched here)
        q.update(seqs or {})
        return L.splitzip_cache_allot(C.byref(_CPool(*[p[x] for x in ("free", "state", "pages", "page", "res")])),
                                      C.byref(_CSeqs(*[q[x] for x in ("table", "starts", "lens", "stride", "n", "rows", "len")])), rows, keep, slots, of, pos, n, None)

    assert call() == -2
    for p in (dict(free=None), dict(state=None), dict(free=buf + 2), dict(state=buf + 1), dict(pages=0), dict(page=4), dict(page=24), dict(page=1 << 31), dict(res=1)):
        assert call(pool=p) == -1, p
    assert call(seqs=dict(n=0)) == 0
    assert call(pool=dict(pages=1 << 31), seqs=dict(n=1)) == -2 and call(seqs=dict(n=1), n=(1 << 30) + 1) == -2
    one = dict(n=1)
    for q in (dict(table=None), dict(starts=None), dict(lens=None), dict(stride=0), dict(table=buf + 2), dict(starts=buf + 1), dict(lens=buf + 2)):
        assert call(seqs={**one, **q}) == -1, q
    for k in (dict(rows=None), dict(rows=buf + 2), dict(keep=buf + 1), dict(slots=buf + 4), dict(of=buf + 2), dict(pos=buf + 1)):
        assert call(seqs=one, **k) == -1, k
    assert L.splitzip_cache_allot(None, None, buf, None, None, None, None, 1, None) == -1
    assert L.splitzip_cache_allot(C.byref(_CPool(buf, buf, 4, 16, 0)), None, buf, None, None, None, None, 1, None) == -1


def of_host(device, **other):
    z = lambda *s, dtype=I32: torch.zeros(*s, dtype=dtype, device=device)   # noqa: E731
    t = dict(free=z(4), state=z(8), table=z(2, 4), starts=z(3), lens=z(2), rows=z(2), keep=z(2), slots=z(5, dtype=I64), row_seqs=z(5), positions=z(5))
    t.update(other)
    return lambda: sz.cache_allot(sz.PagePool(t["free"], t["state"], 16), sz.Sequences(t["table"], t["starts"], t["lens"], 1, 1), t["rows"], t["keep"], t["slots"],
                                  t["row_seqs"], t["positions"])


def test_python_side_checks():
    z = lambda *s, dtype=I32: torch.zeros(*s, dtype=dtype)   # noqa: E731
    for k in (dict(free=z(4).float()), dict(state=z(7)), dict(state=z(16)[::2]), dict(free=z(2, 4)), dict(rows=z(3)), dict(rows=z(2).float()), dict(keep=z(1)),
              dict(keep=z(4)[::2]), dict(slots=z(5)), dict(slots=z(4, dtype=I64)), dict(row_seqs=z(5, dtype=I64)), dict(positions=z(10)[::2]), dict(positions=z(5, 1))):
        with pytest.raises(ValueError, match="must"):
            of_host("cpu", **k)()
    with pytest.raises(ValueError, match="on the GPU"):
        of_host("cpu")()


@pytest.mark.gpu
def test_tensors_that_the_gpu_does_not_reach_are_refused():
    of_host("cuda")()
    for name, t in (("free", torch.zeros(4, dtype=I32)), ("state", torch.zeros(8, dtype=I32)), ("rows", torch.zeros(2, dtype=I32)), ("keep", torch.zeros(2, dtype=I32)),
                    ("slots", torch.zeros(5, dtype=I64)), ("positions", torch.zeros(5, dtype=I32)), ("lens", torch.zeros(2, dtype=I32))):
        with pytest.raises(ValueError, match="on the GPU"):
            of_host("cuda", **{name: t})()
    for k in (dict(rows=torch.zeros(3, dtype=I32, device="cuda")), dict(slots=torch.zeros(4, dtype=I64, device="cuda"))):
        with pytest.raises(ValueError, match="must"):
            of_host("cuda", **k)()


# ---- steps ---------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("n,page,most,room", [(1, 8, 40, 64), (3, 16, 5, 16), (64, 16, 3, 200), (63, 32, 300, 20000), (1024, 8, 9, 12000), (1025, 16, 2, 4096), (3000, 16, 4, 5000),
                                              (2500, 8, 2, 20000)])
def test_many_steps(n, page, most, room):
    """steps of all kinds one behind the other: rows and none, drafts given back, sequences that end and come again, pools that run dry, too many rows"""
    rng = np.random.default_rng(n)
    width = 3 * most // page + 4
    pages = max(4, n * width // 3)
    h = Host(n, width, page, pages, seed=n)
    d = Device(h)
    seen = set()
    for k in range(25):
        rows = rng.integers(-1, most + 1, n) * (rng.random(n) < rng.choice([0.1, 0.6, 1.0]))
        keep = None if k % 5 == 0 else np.where(rng.random(n) < 0.15, rng.integers(-2, 2, n), h.lens - rng.integers(-1, 4, n))
        n_rows = int(np.maximum(rows, 0).sum()) + 3 if k % 7 == 6 else room
        want = h.step(rows, keep, n_rows)
        got = outputs(n_rows)
        sz.cache_allot(d.pool, d.seqs, i32(rows), None if keep is None else i32(keep), *got)
        d.same(h)
        compare(got, want, n_rows)
        seen.add(int(h.state[1]))
    assert 0 in seen


@pytest.mark.gpu
def test_pages_go_back_as_they_lay():
    """drafts that are given back leave the pool as it was, and the next step finds the same pages"""
    h = Host(7, 30, 8, 100, seed=3)
    d = Device(h)
    sz.cache_allot(d.pool, d.seqs, i32([100, 3, 0, 8, 9, 64, 1]))
    lens, free, state = d.lens.clone(), d.free.clone(), d.state.clone()
    first = outputs(80)
    for _ in range(3):
        got = outputs(80)
        sz.cache_allot(d.pool, d.seqs, i32([9, 9, 9, 9, 9, 9, 9]), keep=lens, slots=got[0], row_seqs=got[1], positions=got[2])
        table = d.table.clone()
        if _ == 0:
            first, first_table = got, table
        assert all(torch.equal(a, b) for a, b in zip(first, got)) and torch.equal(first_table, table)
        sz.cache_allot(d.pool, d.seqs, i32([0] * 7), keep=lens)
        assert torch.equal(d.lens, lens) and torch.equal(d.free, free) and int(d.state[0]) == int(state[0])
    sz.cache_allot(d.pool, d.seqs, i32([0] * 7), keep=i32([-1] * 7))
    assert int(d.state[0]) == 100 and sorted(d.free.tolist()) == list(range(100)) and not d.lens.any()
    assert sz.read_pool_state(d.pool)["status"] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n_rows", [100, 5000])
def test_steps_that_cannot_be_taken_change_nothing(n_rows):
    for rows, free, page_tokens, bit in (([60, 20], 2, 8, sz.ALLOT_PAGES), ([n_rows, 1], 40000, 8, sz.ALLOT_ROWS), ([8 * 50 + 1, 0], 100, 8, sz.ALLOT_LENGTH), ([1, 1], -3, 8, sz.ALLOT_POOL)):
        width = 50 if bit == sz.ALLOT_LENGTH else 700
        h = Host(2, width, page_tokens, 40000, free=free)
        h.lens[:] = [0, 0]
        d = Device(h)
        before = [t.clone() for t in (d.table, d.lens, d.free)]
        got = outputs(n_rows)
        sz.cache_allot(d.pool, d.seqs, i32(rows), None, *got)
        h.step(np.array(rows), None, n_rows)
        assert int(h.state[1]) & bit
        d.same(h)
        compare(got, None, n_rows)
        assert all(torch.equal(a, b) for a, b in zip(before, (d.table, d.lens, d.free))) and not d.starts.any()
    s = sz.read_pool_state(d.pool)
    assert s["status"] == sz.ALLOT_POOL and s["free"] == -3 and s["rows"] == 0


@pytest.mark.gpu
def test_the_most_sequences_and_a_long_one():
    n = 65535
    h = Host(n, 1, 8, n + 10, seed=1)
    d = Device(h)
    rows = np.arange(n) % 9
    got = outputs(n * 9)
    want = h.step(rows)
    sz.cache_allot(d.pool, d.seqs, i32(rows), None, *got)
    d.same(h)
    compare(got, want, n * 9)
    # one sequence of a million tokens; a row that only its last token has
    h = Host(3, 70000, 16, 70000, seed=2)
    d = Device(h)
    for rows in ([0, 1 << 20, 0], [5, 1, 0]):
        want = h.step(np.array(rows))
        got = outputs(max(sum(rows), 1) + 100)
        sz.cache_allot(d.pool, d.seqs, i32(rows), None, *got)
        d.same(h)
        compare(got, want, max(sum(rows), 1) + 100)


@pytest.mark.gpu
def test_what_a_program_leaves_out_and_other_streams():
    """any of the outputs, the general way, another stream"""
    results = []
    for leave in ((), (0,), (1, 2), (0, 1, 2)):
        for general in (False, True):
            h = Host(5, 4, 16, 30, seed=4)
            d = Device(h)
            got = [None if k in leave else t for k, t in enumerate(outputs(50))]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            rows = i32([3, 0, 17, 1, 16])
            rows = rows.view(torch.uint32) if general else rows
            want = h.step(np.array([3, 0, 17, 1, 16]))
            torch.cuda.synchronize()
            sz.cache_allot(d.pool, d.seqs, rows, None, *got, stream=side)
            side.synchronize()
            d.same(h)
            for k in range(3):
                if got[k] is not None:
                    compare((got[k],), (want[k],), 50)
            results.append(d.table.cpu())
    assert all(torch.equal(results[0], r) for r in results)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 1500])
def test_lengths_may_be_what_is_kept(n):
    """keep is the tensor of the lengths itself; the most rows hold also where none of the outputs is wanted"""
    h = Host(n, 6, 8, 5 * n, seed=6)
    d = Device(h)
    rows = np.arange(n) % 13
    for _ in range(2):
        want = h.step(rows, h.lens.copy(), 20000)
        got = outputs(20000)
        sz.cache_allot(d.pool, d.seqs, i32(rows), d.lens, *got)
        d.same(h)
        compare(got, want, 20000)
    L, zero = sz.lib(), h.step(np.full(n, 1), None, n - 1)
    assert zero is None
    rows = i32(np.full(n, 1))
    assert L.splitzip_cache_allot(C.byref(d.pool.c), C.byref(d.seqs.c), rows.data_ptr(), None, None, None, None, n - 1, None) == 0
    torch.cuda.synchronize()
    d.same(h)


@pytest.mark.gpu
def test_captured_steps():
    """a step captured once and replayed with other rows, its lengths going on from replay to replay"""
    h = Host(6, 20, 8, 90, seed=5)
    d = Device(h)
    rows, got = i32([0] * 6), outputs(64)
    sz.cache_allot(d.pool, d.seqs, rows, None, *got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sz.cache_allot(d.pool, d.seqs, rows, None, *got)
    rng = np.random.default_rng(5)
    taken = 0
    for _ in range(12):
        now = rng.integers(0, 11, 6)
        rows.copy_(i32(now))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = h.step(now, None, 64)
        d.same(h)
        compare(got, want, 64)
        taken += want is not None
    assert taken > 0


@pytest.mark.gpu
@pytest.mark.parametrize("lens,keep,free,n_rows", [([1 << 30, -9], None, 5, 40), ([2147483647, 30], [5, 2147483647], 5, 40), ([30, 30], [-5, 0], 5, 40), ([30, 30], [0, 0], 2147483647, 40),
                                                   ([30, 30], None, -2147483648, 5000), ([30, 25], [1, 1], 5, 5000), ([0, 0], None, 12, 5000)])
@pytest.mark.parametrize("rows", [[3, 4], [2147483647, 2147483647], [-1, 9]])
def test_calls_stay_in_their_buffers(lens, keep, free, n_rows, rows):
    """whatever lengths, rows, table and state say"""
    g = Guarded()
    h = Host(2, 4, 8, 12, free=free)
    h.lens[:] = lens
    d = Device(h, g)
    got = outputs(n_rows, g)
    sz.cache_allot(d.pool, d.seqs, g(2, dtype=I32, fill=torch.tensor(rows, dtype=I32)), None if keep is None else g(2, dtype=I32, fill=torch.tensor(keep, dtype=I32)), *got)
    assert g.intact()


def test_sizes_that_32_bits_do_not_hold_are_refused():
    """(tensors without memory: nothing looks at more than their sizes)"""
    large = lambda dtype: torch.empty((1 << 32) + 5, dtype=dtype, device="meta")   # noqa: E731
    for k in (dict(slots=large(I64), row_seqs=None, positions=None), dict(slots=None, row_seqs=large(I32), positions=None), dict(slots=None, row_seqs=None, positions=large(I32)),
              dict(free=torch.empty((1 << 32) + 4, dtype=I32, device="meta"))):
        with pytest.raises(ValueError, match="must have"):
            of_host("cpu", **k)()
    z = torch.zeros(8, dtype=I32)
    for page in ((1 << 32) + 16, -16):
        with pytest.raises(ValueError, match="must be"):
            sz.PagePool(z, z, page)
