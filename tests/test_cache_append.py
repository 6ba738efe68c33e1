"""A step's projections (splitzip_cache_append) against their formulas in 64 bits.

What a value is off in front of its last rounding, in 32 bits, each operation 2^-24 of its result at most: a norm's sum of squares, all of one sign, goes
through 8 + 5 additions (half of that in the root), its mean, root, the root's inverse (2^-22) and three products: 2^-20 of the
value.  A sine or cosine is off by its argument's rounding (a turn of 1/2 in 24 bits, 2^-23), by what 2^30 turns leave of 53 bits
(2^-22) and by its own (2^-22): 2^-20.  Two products and a sum: (|a| + |b|) 2^-18 |scaling| bounds all of it.  Then one rounding: half a step of
the words, which for those of the cache is a step of the grid that the scale byte says; and a byte is that of the largest magnitude or, where that is nearer to
a border than its error, the next one's."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz
from paper_2605_01708_amd.binding import _CCache, _CRotation, _CSeqs
from test_cache_guards import Guarded

I32 = torch.int32
KINDS = [sz.BF16, sz.FP8_E5M2, sz.FP8_E4M3, sz.FP4_E2M1]
GRID = {sz.FP8_E5M2: (57344.0, 2, -14), sz.FP8_E4M3: (448.0, 3, -6), sz.FP4_E2M1: (6.0, 1, 0)}   # largest word, mantissa bits, least exponent


class Step:
    def __init__(self, kind, lens, rows, q_heads=4, heads=2, dim=128, page=16, seed=0, make=None):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.kind, self.lens, self.rows, self.q_heads, self.heads, self.dim, self.page = kind, lens, rows, q_heads, heads, dim, page
        used = [-(-max(n, 1) // page) for n in lens]
        self.pages = sum(used) + 2
        order = np.random.default_rng(seed).permutation(self.pages)
        self.table, at = np.zeros((len(lens), max(used)), np.int32), 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at:at + u]
            at += u
        self.n = sum(rows)
        word = {sz.BF16: (dim, torch.bfloat16), sz.FP4_E2M1: (dim // 2, torch.uint8)}.get(kind, (dim, torch.uint8))
        make = make or (lambda *s, dtype, fill=None: torch.zeros(*s, dtype=dtype, device="cuda") if fill is None else torch.as_tensor(fill, device="cuda").to(dtype).contiguous())
        self.kv = [make(self.pages, page, heads, word[0], dtype=word[1], fill=torch.full((self.pages, page, heads, word[0]), 3)) for _ in range(2)]
        groups = (dim // 32,) if kind == sz.FP4_E2M1 else ()
        self.scales = [None if kind == sz.BF16 else make(self.pages, heads, *groups, page, dtype=torch.uint8, fill=torch.full((self.pages, heads, *groups, page), 9)) for _ in range(2)]
        self.cache = sz.KvCache(*self.kv, kind, *self.scales)
        self.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.dev = [make(*self.table.shape, dtype=I32, fill=torch.from_numpy(self.table)), make(len(rows) + 1, dtype=I32, fill=torch.from_numpy(self.starts)),
                    make(len(lens), dtype=I32, fill=torch.tensor(lens, dtype=I32))]
        self.seqs = sz.Sequences(*self.dev, max_rows=max(rows), max_len=max(lens))
        # as one tensor of projections
        total = q_heads + 2 * heads
        self.qkv = make(self.n, total, dim, dtype=torch.bfloat16, fill=torch.randn(self.n, total, dim, generator=gen, device="cuda") * torch.exp(torch.randn(total, dim, generator=gen, device="cuda")))
        self.q, self.k, self.v = self.qkv[:, :q_heads], self.qkv[:, q_heads:q_heads + heads], self.qkv[:, q_heads + heads:]
        self.q_out = make(self.n, q_heads, dim, dtype=torch.bfloat16)
        self.k_out = make(self.n, heads, dim, dtype=torch.bfloat16)

    def where(self):
        """of every row: position, page, place; page -1: in front of the sequence"""
        out = []
        for s, (n, T) in enumerate(zip(self.lens, self.rows)):
            for i in range(T):
                t = n - T + i
                out.append((t, int(self.table[s, t // self.page]) if t >= 0 else -1, t % self.page))
        return np.array(out).T

    def cached(self, which):
        """values that the cache holds for the rows, in 64 bits, [rows, heads, dim], and powers of the scales, [rows, heads, groups]"""
        _, page, place = self.where()
        words = self.kv[which].cpu()[page, place]
        if self.kind == sz.BF16:
            return words.double().numpy(), None
        b = self.scales[which].cpu().movedim(-1, 1)[page, place].numpy().astype(np.int64)
        b = b if self.kind == sz.FP4_E2M1 else b[..., None]
        if self.kind == sz.FP4_E2M1:
            nibble = torch.stack([words & 15, words >> 4], -1).flatten(-2).numpy()
            x = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6])[nibble]
        else:
            x = words.view(torch.float8_e5m2 if self.kind == sz.FP8_E5M2 else torch.float8_e4m3fn).double().numpy()
        p = np.exp2(b - 127.0)
        return x * np.repeat(p, self.dim // p.shape[-1], -1), b


def turned(x, weight, offset, eps, freqs, positions, interleaved, scaling):
    """a head's formulas in 64 bits, and what 32 bits may leave them off"""
    x = x.double().cpu().numpy()
    if eps is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * (weight.double().cpu().numpy() + offset)
    off = np.abs(x) * 2.0 ** -20 * (eps is not None)
    if freqs is not None:
        f = freqs.double().cpu().numpy()
        half = len(f)
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        t = (np.asarray(positions, float)[:, None] * f)[:, None]
        u, w = x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = scaling * (u * np.cos(t) - w * np.sin(t)), scaling * (w * np.cos(t) + u * np.sin(t))
        off[..., a] = off[..., b] = (np.abs(u) + np.abs(w)) * 2.0 ** -18 * abs(scaling)
    return x, off


def near(got, x, off):
    assert (np.abs(got - x) <= 2.0 ** -8 * (np.abs(x) + off) + off).all(), np.abs(got - x).max()


def check_cached(step, which, x, off):
    got, b = step.cached(which)
    if step.kind == sz.BF16:
        return near(got, x, off)
    largest, bits, least = GRID[step.kind]
    groups = b.shape[-1]
    width = step.dim // groups
    top, slack = (np.abs(x).reshape(*b.shape, width).max(-1), off.reshape(*b.shape, width).max(-1))
    powers = largest * np.exp2(np.arange(255) - 127.0)
    low, high = (np.searchsorted(powers, y) for y in (np.maximum(top - slack, 0), top + slack))
    assert ((low <= b) & (b <= high)).all()
    p = np.repeat(np.exp2(b - 127.0), width, -1)
    y = (np.abs(x) + off) / p
    unit = np.exp2(np.maximum(np.floor(np.log2(np.maximum(y, 2.0 ** -40))), least) - bits)
    assert (np.abs(got - x) <= p * unit / 2 + off).all()


def call(step, how, q_out=None, k_out=None, **k):
    sz.cache_append(step.q, step.k, step.v, step.cache, step.seqs, how, step.q_out if q_out is None else q_out, k_out, **k)
    torch.cuda.synchronize()


def check(step, q_out, k_out, weights, offset, eps, freqs, interleaved, scaling, positions=None):
    at, page, _ = step.where()
    positions = at if positions is None else positions
    q, q_off = turned(step.qkv0[:, :step.q_heads], weights[0], offset, eps, freqs, positions, interleaved, scaling)
    k, k_off = turned(step.qkv0[:, step.q_heads:step.q_heads + step.heads], weights[1], offset, eps, freqs, positions, interleaved, scaling)
    v = step.qkv0[:, step.q_heads + step.heads:].double().cpu().numpy()
    near(q_out.double().cpu().numpy(), q, q_off)
    if k_out is not None:
        near(k_out.double().cpu().numpy(), k, k_off)
    there = page >= 0
    for which, x, off in ((0, k, k_off), (1, v, np.zeros_like(v))):
        kept = Step.cached(step, which)
        full = step.cached
        step.cached = lambda w, kept=kept: (kept[0][there], None if kept[1] is None else kept[1][there])
        check_cached(step, which, x[there], off[there])
        step.cached = full


def freqs_of(half, base=10000.0):
    return (base ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))).float() if half else None


# ---- what is refused -----------------------------------------------------------------------------------

def test_descriptions_are_checked():
    L, buf = sz.lib(), 1 << 16

    def call(n=1, q=buf, qs=512, qo=buf, qos=512, k=buf, ks=256, v=buf, vs=256, ko=None, kos=0, heads=4, cache=None, seqs=None, **how):
        c = dict(k=buf, v=buf, ks=buf, vs=buf, dtype=sz.FP8_E5M2, heads=2, dim=128, page=16, pages=4, res=0, ps=16 * 256, ts=256, hs=128, ss=32)
        c.update(cache or {})
        c = _CCache(*[c[x] for x in ("k", "v", "ks", "vs", "dtype", "heads", "dim", "page", "pages", "res", "ps", "ts", "hs", "ss")])
        h = dict(f=buf, qw=buf, kw=buf, pos=None, scaling=1.0, eps=1e-6, off=0.0, rot=128, inter=0, norm=1, f32=0, res=0)
        h.update(how)
        h = _CRotation(*[h[x] for x in ("f", "qw", "kw", "pos", "scaling", "eps", "off", "rot", "inter", "norm", "f32", "res")])
        return L.splitzip_cache_append(C.byref(c), C.byref(seqs or _CSeqs(buf, buf, buf, 4, 2, 1, 64)), C.byref(h), q, qs, qo, qos, k, ks, v, vs, ko, kos, n, heads, None)

    assert call(n=0) == 0
    for k in (dict(rot=120), dict(rot=144), dict(f=None), dict(f=buf + 2), dict(inter=2), dict(norm=2), dict(f32=2), dict(res=1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
              dict(eps=float("inf")), dict(eps=1e-40), dict(qw=buf + 8), dict(kw=buf + 2), dict(pos=buf + 2), dict(cache=dict(dim=96)), dict(cache=dict(k=None))):
        assert call(n=0, **k) == (-2 if k.get("cache", {}).get("dim") == 96 else -1), k
    assert call(n=0, rot=0, f=None) == 0 and call(n=0, norm=0, eps=0.0, qw=None, kw=None) == 0 and call(n=0, rot=16) == 0
    for k in (dict(q=None), dict(qs=504), dict(qs=516), dict(qo=None), dict(qos=511), dict(k=None), dict(v=buf + 8), dict(ks=248), dict(vs=252), dict(ko=buf + 2, kos=256), dict(ko=buf, kos=128),
              dict(qos=520), dict(ko=buf, kos=264)):                     # (in place needs one stride)
        assert call(**k) == -1, k
    assert call(n=(1 << 30) + 1) == -2 and call(heads=(1 << 23) + 1, qs=1 << 31, qos=1 << 31) == -2
    assert call(seqs=_CSeqs(None, None, None, 0, 0, 0, 0)) == 0 and call(seqs=_CSeqs(buf, buf, buf, 4, 1 << 16, 1, 64)) == -2
    assert L.splitzip_cache_append(None, None, None, *[None, 0] * 5, 0, 0, None) == -1


def test_python_side_checks():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)   # noqa: E731
    for k in (dict(freqs=z(64)), dict(freqs=z(8, 8, dtype=torch.float32)), dict(freqs=z(64, dtype=torch.float32)[::2]), dict(q_weight=z(128)), dict(eps=1e-6, q_weight=z(128), k_weight=z(64)),
              dict(eps=1e-6, q_weight=z(128), k_weight=z(128, dtype=torch.float32)), dict(eps=1e-6, q_weight=z(128, dtype=torch.float16)), dict(positions=z(4)),
              dict(eps=1e-6, k_weight=z(256)[::2]), dict(positions=z(8, dtype=I32)[::2])):
        with pytest.raises(ValueError):
            sz.Rotation(**k)
    c, s = sz.KvCache(z(3, 16, 2, 64), z(3, 16, 2, 64), sz.BF16), sz.Sequences(z(2, 4, dtype=I32), z(3, dtype=I32), z(2, dtype=I32), 1, 64)
    q, k, how = z(5, 4, 64), z(5, 2, 64), sz.Rotation()
    for a in ((q, k, k, how, None), (None, k, k, how, q), (q[0], k, k, how, q[0]), (q, k, k[:4], how, q), (q, k, k, how, q[:4]), (q, k, k, how, z(5, 2, 64)), (q[:4], k, k, how, q[:4]),
              (q.float(), k, k, how, q), (q, k.transpose(0, 1), k, how, q), (q, k, k, sz.Rotation(eps=1e-6, q_weight=z(128)), q), (q, k, k, sz.Rotation(positions=z(4, dtype=I32)), q)):
        with pytest.raises(ValueError, match="must|go together"):
            sz.cache_append(a[0], a[1], a[2], c, s, a[3], a[4])
    with pytest.raises(ValueError, match="must"):
        sz.cache_append(q, k, k, c, s, how, q, k_out=z(5, 4, 64))
    with pytest.raises(ValueError, match="on the GPU"):
        sz.cache_append(q, k, k, c, s, how, q)


@pytest.mark.gpu
def test_the_short_way_refuses_what_the_general_way_refuses():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")   # noqa: E731
    c, s = sz.KvCache(z(3, 16, 2, 64), z(3, 16, 2, 64), sz.BF16), sz.Sequences(z(2, 4, dtype=I32), z(3, dtype=I32), z(2, dtype=I32), 1, 64)
    q, k, how = z(5, 4, 64), z(5, 2, 64), sz.Rotation()
    sz.cache_append(q, k, k, c, s, how, q)
    for a in ((q, k, k[:4], how, q, None), (q, k, k, how, q[:4], None), (q, k, k, how, z(5, 2, 64), None), (q, k, k, sz.Rotation(eps=1e-6, k_weight=z(128)), q, None),
              (q, k, k, sz.Rotation(positions=z(4, dtype=I32)), q, None), (q, k, k, how, q, z(4, 2, 64)), (None, k, k, how, q, None), (q, k, k, how, None, None),
              (None, k, k, sz.Rotation(positions=z(4, dtype=I32)), None, None), (q, k.cpu(), k, how, q, None), (q, k, k, sz.Rotation(torch.zeros(8)), q, None)):
        with pytest.raises(ValueError):
            sz.cache_append(a[0], a[1], a[2], c, s, a[3], a[4], a[5])


# ---- values --------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,rotary,q_heads,heads", [(128, 128, 4, 2), (64, 64, 5, 3), (256, 256, 2, 1), (128, 64, 8, 8), (256, 48, 3, 1), (64, 16, 1, 1), (128, 96, 40, 2), (128, 112, 7, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norms_and_rotations(kind, dim, rotary, q_heads, heads, interleaved):
    st = Step(kind, [37, 1, 100, 3, 16], [37, 1, 13, 0, 2], q_heads, heads, dim, seed=dim + rotary)
    st.qkv0 = st.qkv.clone()
    weights = [(1 + 0.3 * torch.randn(dim, device="cuda", generator=torch.Generator("cuda").manual_seed(i))).to(torch.bfloat16) for i in range(2)]
    freqs = freqs_of(rotary // 2)
    call(st, sz.Rotation(freqs, interleaved, 1.0, 1e-6, *weights), k_out=st.k_out)
    assert torch.equal(st.qkv, st.qkv0)
    check(st, st.q_out, st.k_out, weights, 0.0, 1e-6, freqs, interleaved, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [sz.BF16, sz.FP4_E2M1])
@pytest.mark.parametrize("eps,weighted,offset,rotary,scaling,dtype", [(None, False, 0.0, 128, 1.0, None), (1e-5, False, 0.0, 0, 1.0, None), (1e-5, True, 1.0, 128, 1.3, torch.float32),
                                                                      (0.5, True, 0.25, 64, -0.7, torch.bfloat16), (1e-6, True, 0.0, 0, 1.0, torch.float32)])
def test_options(kind, eps, weighted, offset, rotary, scaling, dtype):
    st = Step(kind, [50, 60], [3, 60], seed=1)
    st.qkv0 = st.qkv.clone()
    weights = [0.5 * torch.randn(128, device="cuda", dtype=torch.float32).to(dtype) if weighted else None for _ in range(2)]
    if weighted and dtype == torch.float32:
        weights[0] = None                                         # of K alone
    freqs = freqs_of(rotary // 2, 500000.0)
    call(st, sz.Rotation(freqs, False, scaling, eps, *weights, weight_offset=offset))
    check(st, st.q_out, None, weights, offset, eps, freqs, False, scaling)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_without_norm_and_rotation_it_writes(kind, dim):
    """the words, scales and rows of cache_write, bit for bit, special values among them; rows in front of token 0, and what no row is written to, as they were"""
    from test_cache_fp4 import special_groups

    a, b = (Step(kind, [37, 5, 0, 70], [37, 7, 0, 20], 3, 2, dim, seed=2) for _ in range(2))
    x = torch.from_numpy(special_groups(a.n, 7, dim, 5)).to(torch.bfloat16).cuda()
    for st in (a, b):
        st.qkv.copy_(x)
    call(a, sz.Rotation())
    sz.cache_write(b.k, b.v, b.cache, b.seqs)
    assert torch.equal(a.q_out.view(torch.int16), a.q.contiguous().view(torch.int16)) or torch.equal(torch.nan_to_num(a.q_out, 5.0), torch.nan_to_num(a.q, 5.0))
    for p, q in zip(a.kv + a.scales, b.kv + b.scales):
        assert p is None or torch.equal(p.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.gpu
def test_far_positions():
    """positions up to 2^30, also below 0, and given ones: the angle is exact where 32 bits of it would not be"""
    st = Step(sz.BF16, [9, 4], [9, 4], seed=3)
    st.qkv0 = st.qkv.clone()
    pos = [(1 << 30) - 1, 1 << 30, -(1 << 30), 0, 1, -1, 16777217, 123456789, 1000003, 7, 65537, -40000, 999999999]
    for interleaved in (False, True):
        freqs = freqs_of(64)
        call(st, sz.Rotation(freqs, interleaved, positions=torch.tensor(pos, dtype=I32, device="cuda")), k_out=st.k_out)
        check(st, st.q_out, st.k_out, (None, None), 0.0, None, freqs, interleaved, 1.0, pos)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [sz.BF16, sz.FP8_E4M3, sz.FP4_E2M1])
def test_long_calls_are_short_ones(kind):
    """many rows of many heads, and the same rows one sequence at a time: the same bits, whatever the launch is cut for"""
    lens, rows = [3000, 40, 1, 900], [2500, 40, 1, 0]
    a, b = (Step(kind, lens, rows, 32, 8, 128, seed=4) for _ in range(2))
    freqs = freqs_of(64)
    w = torch.rand(128, device="cuda") + 0.5
    how = sz.Rotation(freqs, False, 1.0, 1e-6, w, w)
    call(a, how)
    for s in range(3):
        cut = slice(int(b.starts[s]), int(b.starts[s + 1]))
        seqs = sz.Sequences(b.dev[0][s:s + 1].contiguous(), torch.tensor([0, rows[s]], dtype=I32, device="cuda"), b.dev[2][s:s + 1].contiguous(), 1, 1)
        sz.cache_append(b.q[cut], b.k[cut], b.v[cut], b.cache, seqs, how, b.q_out[cut])
    torch.cuda.synchronize()
    assert torch.equal(a.q_out, b.q_out)
    for p, q in zip(a.kv + a.scales, b.kv + b.scales):
        assert p is None or torch.equal(p, q)
    a.qkv0 = a.qkv
    check(a, a.q_out, None, (w, w), 0.0, 1e-6, freqs, False, 1.0)


@pytest.mark.gpu
def test_in_place_without_q_other_streams_and_graphs():
    st = Step(sz.FP8_E5M2, [300, 70], [3, 2], seed=6)
    freqs = freqs_of(64)
    how = sz.Rotation(freqs, False, 1.0, 1e-6)
    first = st.qkv.clone()
    call(st, how, k_out=st.k_out)
    want = [t.clone() for t in (st.q_out, st.k_out, *st.kv, *st.scales)]
    # in place, on another stream
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sz.cache_append(st.q, st.k, st.v, st.cache, st.seqs, how, st.q, st.k, stream=side)
    side.synchronize()
    assert torch.equal(st.q, want[0]) and torch.equal(st.k, want[1]) and all(torch.equal(a, b) for a, b in zip((*st.kv, *st.scales), want[2:]))
    # no Q
    st.qkv.copy_(first)
    for t in st.kv:
        t.fill_(3)
    sz.cache_append(None, st.k, st.v, st.cache, st.seqs, how, None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*st.kv, *st.scales), want[2:]))
    # captured, and replayed at other lengths and positions
    pos = torch.zeros(5, dtype=I32, device="cuda")
    how = sz.Rotation(freqs, False, positions=pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sz.cache_append(st.q, st.k, st.v, st.cache, st.seqs, how, st.q_out)
    for k, lens in enumerate(([300, 70], [3, 2], [17, 64], [300, 70])):
        st.lens = lens
        st.dev[2].copy_(torch.tensor(lens, dtype=I32))
        pos.copy_(torch.arange(5, device="cuda") * 1000 * k)
        st.qkv.copy_(first * (k + 1))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        st.qkv0 = st.qkv
        check(st, st.q_out, None, (None, None), 0.0, None, freqs, False, 1.0, [1000 * k * i for i in range(5)])


@pytest.mark.gpu
def test_the_short_way_and_the_general_way(monkeypatch):
    a, b = (Step(sz.FP4_E2M1, [300, 70], [3, 2], seed=7) for _ in range(2))
    how = sz.Rotation(freqs_of(64), True, 1.0, 1e-6)
    f, taken = sz.lib().fast_cache.splitzip_cache_append, []
    monkeypatch.setattr(sz.lib().fast_cache, "splitzip_cache_append", lambda *x: taken.append(f(*x)) or taken[-1])
    call(a, how, k_out=a.k_out)
    assert taken == [0]
    monkeypatch.setattr(sz.lib().fast_cache, "splitzip_cache_append", lambda *x: 1)
    call(b, how, k_out=b.k_out)
    for p, q in zip((a.q_out, a.k_out, *a.kv, *a.scales), (b.q_out, b.k_out, *b.kv, *b.scales)):
        assert torch.equal(p, q)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,starts,table", [((40, 50), (0, 20, 40), None), ((1 << 30, -5), (0, 20, 40), None), ((40, 50), (-3, 2, 1 << 20), None), ((40, 50), (3, 1, 4), None), ((40, 50), (0, 20, 40), -1)])
def test_calls_stay_in_their_buffers(kind, lens, starts, table):
    g = Guarded()
    st = Step(kind, [40, 50], [20, 20], 5, 2, 64, seed=8, make=g)
    st.dev[2].copy_(torch.tensor(lens, dtype=I32))
    st.dev[1].copy_(torch.tensor(starts, dtype=I32))
    if table is not None:
        st.dev[0].fill_(table)
    freqs = g(24, dtype=torch.float32, fill=torch.rand(24))
    w = g(64, dtype=torch.float32, fill=torch.rand(64))
    call(st, sz.Rotation(freqs, False, 1.0, 1e-6, w, w, positions=g(40, dtype=I32, fill=torch.arange(40))), k_out=st.k_out)
    assert g.intact()


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", [sz.BF16, sz.FP8_E4M3])
def test_norms_of_the_largest_magnitudes(kind, dim):
    """elements of 2^60, all of them, some of them, and of what is next to nothing beside them"""
    st = Step(kind, [20], [5], 3, 2, dim, seed=9)
    big = 2.0 ** 60 * torch.where(torch.randn(st.qkv.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(9)) > 0, 1.0, -1.0)
    big[1, :, 1::2] = 0.0
    big[2, :, 1:] = 2.0 ** -60
    big[3] *= 2.0 ** -9
    st.qkv.copy_(big)
    st.qkv0 = st.qkv.clone()
    for eps in (1e-6, 2.0 ** -126):
        call(st, sz.Rotation(eps=eps), k_out=st.k_out)
        check(st, st.q_out, st.k_out, (None, None), 0.0, eps, None, False, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_v_is_written_as_it_is(kind):
    """every BF16 word: what cache_write makes of it, bit for bit, whatever K's norm and rotation are"""
    a, b = (Step(kind, [200], [160], 3, 4, 128, seed=10) for _ in range(2))
    words = torch.arange(65536, dtype=I32, device="cuda")
    rows = torch.cat([words.view(128, 4, 128), words.view(-1, 128).T.reshape(-1)[:32 * 512].view(32, 4, 128)]).to(torch.int16)   # alike in size, and mixed
    for st in (a, b):
        st.v.view(torch.int16).copy_(rows)
    call(a, sz.Rotation(freqs_of(64), eps=1e-6))
    sz.cache_write(b.k, b.v, b.cache, b.seqs)
    torch.cuda.synchronize()
    x, y = a.kv[1], b.kv[1]
    if kind != sz.BF16:
        assert torch.equal(a.scales[1], b.scales[1])
    if kind == sz.FP4_E2M1:                                          # (words under the byte 255 are not looked at)
        fine = (a.scales[1] != 255).movedim(-1, 1).repeat_interleave(16, -1)
        x, y = x[fine], y[fine]
    assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_positions_are_one_for_each_row():
    for t in (torch.zeros(5, 2, dtype=I32), torch.zeros((), dtype=I32)):
        with pytest.raises(ValueError, match="positions"):
            sz.Rotation(positions=t)
