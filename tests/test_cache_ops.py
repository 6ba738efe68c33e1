"""The cache operators (splitzip_cache_write / _read / _attention / _move) against their formulas in 64 bits.

Words and scale bytes are exact: a power of two is found and one rounding is made, so nothing may differ.  Attention's tolerance:
the result is rounded to BF16 (8 significant bits: 2^-8 of it at most), every weight was (2^-8 of the mean of |v| under the weights, A), and
a score's error dx -- a dot product of D terms in 32 bits, at most (D + 8) 2^-23 sum |q k| scale, the cap's 4e-7 of it and the
bias's own rounding -- moves a weight by 2 dx at most, its maximum and itself."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2605_01708_amd as sz
from paper_2605_01708_amd.binding import _CAttention, _CCache, _CSeqs

KINDS = [sz.BF16, sz.FP8_E5M2, sz.FP8_E4M3]
FLOATS = {sz.BF16: torch.bfloat16, sz.FP8_E5M2: torch.float8_e5m2, sz.FP8_E4M3: torch.float8_e4m3fn}
FORMAT = {sz.BF16: (7, -126, 127), sz.FP8_E5M2: (2, -14, 15), sz.FP8_E4M3: (3, -6, 8)}   # mantissa bits, least and largest exponent


def rounded(x, kind):
    """values in 64 bits to the nearest of the format, ties to even"""
    bits, least, _ = FORMAT[kind]
    e = np.maximum(np.frexp(x)[1] - 1, least)
    unit = np.ldexp(1.0, e - bits)
    with np.errstate(invalid="ignore"):
        y = np.where(np.isfinite(x), np.rint(x / unit) * unit, x)
        return np.where(np.abs(y) >= 2.0 ** 128, np.sign(y) * np.inf, y) if kind == sz.BF16 else y


def scale_byte(row, kind):
    a = np.abs(row[np.isfinite(row)]).max(initial=0.0)
    for b in range(255):
        if a <= 1.75 * 2.0 ** (FORMAT[kind][2] + b - 127):
            return b
    raise AssertionError


def quantised(x, kind):
    """x [..., D] in 64 bits: word values and bytes"""
    flat = x.reshape(-1, x.shape[-1])
    bytes_ = np.array([scale_byte(r, kind) for r in flat], np.uint8)
    y = rounded(flat * np.ldexp(1.0, 127 - bytes_.astype(int))[:, None], kind)
    if kind == sz.FP8_E4M3:
        y = np.where(np.isinf(y), np.nan, y)
    return y.reshape(x.shape), bytes_.reshape(x.shape[:-1])


class World:
    """Sequences with cached tokens in a pool of shuffled pages, on the device and, as values in 64 bits, here.

    layout "nhd": [pages, tokens, heads, dim]; "hnd": heads outside the tokens; "side": K and V of a page side by side;
    "flat": no table, sequence s is page s."""

    def __init__(self, kind, lens, rows, heads=2, dim=128, page=16, layout="nhd", seed=0, words=None, max_rows=None, max_len=None, junk=True,
                 device="cuda"):
        rng = np.random.default_rng(seed)
        self.kind, self.lens, self.rows, self.heads, self.dim, self.page = kind, lens, rows, heads, dim, page
        n, es = len(lens), 2 if kind == sz.BF16 else 1
        if layout == "flat":
            page = self.page = max(8, -(-max(lens, default=1) // 8) * 8)
            self.pages, table = max(n, 1), None
        else:
            used = [-(-x // page) for x in lens]
            self.pages = sum(used) + 2
            order = rng.permutation(self.pages)
            table, at = np.full((n, max(max(used, default=1), 1)), 1 << 30, np.int32), 0
            for s, u in enumerate(used):
                table[s, :u] = order[at:at + u]
                at += u
        self.table = table
        x = rng.standard_normal((2, self.pages, page, heads, dim)) * np.exp(0.5 * rng.standard_normal((2, 1, 1, heads, dim)))
        self.scales = None
        if kind == sz.BF16:
            self.value = rounded(x, kind)
            raw = torch.from_numpy(self.value).to(torch.bfloat16).view(torch.int16)
        else:
            w, b = quantised(x, kind)
            self.value = w * np.ldexp(1.0, b.astype(int) - 127)[..., None]
            raw = torch.from_numpy(w).to(FLOATS[kind]).view(torch.uint8)
            self.scales = torch.from_numpy(b).permute(0, 1, 3, 2).contiguous().to(device)
        # what belongs to no token may hold anything
        owned = np.zeros((self.pages, page), bool)
        for s in range(n):
            for t in range(lens[s]):
                owned[self.slot(s, t)] = True
        if junk:
            bad = {sz.BF16: 0x7fc0, sz.FP8_E5M2: 0x7f, sz.FP8_E4M3: 0x7f}[kind]
            raw[:, torch.from_numpy(~owned)] = bad
        if layout == "hnd":
            pool = raw.permute(0, 1, 3, 2, 4).contiguous().to(device)
            k, v = pool[0].transpose(1, 2), pool[1].transpose(1, 2)
        elif layout == "side":
            pool = raw.permute(1, 0, 2, 3, 4).contiguous().to(device)
            k, v = pool[:, 0], pool[:, 1]
        else:
            pool = raw.to(device)
            k, v = pool[0], pool[1]
        assert es == k.element_size()
        self.owned, self.pool = owned, pool
        self.cache = sz.KvCache(k, v, kind, *([None, None] if self.scales is None else self.scales))
        starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.starts, self.n_rows = starts, int(starts[-1])
        self.dev = [None if table is None else torch.from_numpy(table).to(device), torch.from_numpy(starts).to(device),
                    torch.tensor(lens, dtype=torch.int32, device=device)]
        self.seqs = sz.Sequences(*self.dev, max_rows=max(rows, default=0) if max_rows is None else max_rows,
                                 max_len=max(lens, default=0) if max_len is None else max_len)

    def slot(self, s, t):
        return (s, t) if self.table is None else (int(self.table[s, t // self.page]), t % self.page)

    def set(self, s, t, which, head, values):
        """words of a token replaced on the device (BF16 alone) and here"""
        p, a = self.slot(s, t)
        self.value[which, p, a, head] = values
        (self.cache.k, self.cache.v)[which].view(torch.bfloat16)[p, a, head] = torch.from_numpy(np.asarray(values)).to(torch.bfloat16)

    def tokens(self, s, n):
        """K and V of the first n tokens, [2, n, heads, dim]"""
        at = [self.slot(s, t) for t in range(n)]
        p, a = np.array([x[0] for x in at], int), np.array([x[1] for x in at], int)
        return self.value[:, p, a]


def attend(w, q, scale, softcap=0.0, window=0, slopes=None, see=None, positions=None):
    """out, lse and the tolerances' A and dx, in 64 bits; see(s, i, j): row i sees row j of its sequence"""
    heads = q.shape[1]
    group = heads // w.heads
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    mean, dx = np.zeros(q.shape), np.zeros(q.shape[:2])
    for s, (n, T) in enumerate(zip(w.lens, w.rows)):
        if not T or not n:
            continue
        k, v = w.tokens(s, n)
        base = n - T
        for i in range(T):
            row = w.starts[s] + i
            where = lambda r: base + r if positions is None else int(positions[w.starts[s] + r])   # noqa: E731
            pos = np.array([t if t < base else where(t - base) for t in range(n)])
            ok = np.array([t < base or bool(t - base <= i if see is None else see(s, i, t - base)) for t in range(n)])
            if window:
                ok &= where(i) - pos < window
            if not ok.any():
                continue
            for h in range(heads):
                kk, vv = k[ok, h // group], v[ok, h // group]
                x = scale * (kk @ q[row, h])
                err = (w.dim + 8) * 2.0 ** -23 * scale * (np.abs(kk) @ np.abs(q[row, h]))
                if softcap:
                    x = softcap * np.tanh(x / softcap)
                    err = err + 4e-7 * softcap
                if slopes is not None:
                    x = x + slopes[h] * (pos[ok] - where(i))
                err = err + 2.0 ** -21 * np.abs(x)
                top = x.max()
                p = np.exp(x - top)
                out[row, h] = p @ vv / p.sum()
                lse[row, h] = top + math.log(p.sum())
                mean[row, h] = p @ np.abs(vv) / p.sum()
                dx[row, h] = err.max()
    return out, lse, mean, dx


def close(got, got_lse, want):
    out, lse, mean, dx = want
    got, got_lse = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    bound = 2.0 ** -8 * 1.01 * np.abs(out) + (2.0 ** -8 * 1.01 + 2.5 * dx[..., None] + 2.0 ** -20) * mean
    assert np.isfinite(got).all()
    worst = np.abs(got - out) - bound
    assert (worst <= 0).all(), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    assert (np.isneginf(lse) == np.isneginf(got_lse)).all()
    fine = np.isfinite(lse)
    assert (np.abs(got_lse[fine] - lse[fine]) <= dx[fine] + 2.0 ** -20 * (1 + np.abs(lse[fine]))).all()


def queries(w, group, seed=5):
    q = rounded(np.random.default_rng(seed).standard_normal((w.n_rows, w.heads * group, w.dim)), sz.BF16)
    return q, torch.from_numpy(q).to(torch.bfloat16).cuda()


def run(w, qd, how, out=None):
    out = torch.full_like(qd, float("nan")) if out is None else out
    lse = torch.full(qd.shape[:2], float("nan"), device="cuda")
    ws = sz.attention_workspace(w.cache, w.seqs, qd.shape[0], qd.shape[1])
    ws.fill_(255)
    sz.cache_attention(qd, w.cache, w.seqs, out, ws, how, lse)
    torch.cuda.synchronize()
    return out, lse


def random_tree(T, rng, words):
    """ancestor bits [T, words] and depths of a random tree, its root row 0"""
    bits, depth = [1], [0]
    for i in range(1, T):
        p = int(rng.integers(max(0, i - 7), i))
        bits.append(bits[p] | 1 << i)
        depth.append(depth[p] + 1)
    out = np.array([[b >> 64 * k & (1 << 64) - 1 for k in range(words)] for b in bits], np.uint64).view(np.int64)
    return out, depth, bits


# ---- what is refused -----------------------------------------------------------------------------------

def test_descriptions_are_checked():
    L, buf = sz.lib(), 1 << 16

    def cache(**k):
        d = dict(k=buf, v=buf, ks=buf, vs=buf, dtype=sz.FP8_E5M2, heads=8, dim=128, page=16, pages=4, res=0, ps=16 * 1024, ts=1024, hs=128, ss=128)
        d.update(k)
        return _CCache(*[d[x] for x in ("k", "v", "ks", "vs", "dtype", "heads", "dim", "page", "pages", "res", "ps", "ts", "hs", "ss")])

    def seqs(**k):
        d = dict(table=buf, starts=buf, lens=buf, stride=4, n=2, rows=1, len=64)
        d.update(k)
        return _CSeqs(*[d[x] for x in ("table", "starts", "lens", "stride", "n", "rows", "len")])

    def how(**k):
        d = dict(scale=1.0, cap=0.0, slopes=None, tree=None, pos=None, words=0, window=0, res=0)
        d.update(k)
        return _CAttention(*[d[x] for x in ("scale", "cap", "slopes", "tree", "pos", "words", "window", "res")])

    def write(c=None, q=None, k=buf, ks=1024, v=buf, vs=1024, n=0):
        return L.splitzip_cache_write(C.byref(cache() if c is None else c), C.byref(seqs() if q is None else q), k, ks, v, vs, n, None)

    def attention(c=None, q=None, h=None, qa=buf, qs=4096, out=buf, os=4096, lse=None, n=0, heads=32, ws=buf, wsb=1 << 30):
        return L.splitzip_cache_attention(C.byref(cache() if c is None else c), C.byref(seqs() if q is None else q), C.byref(how() if h is None else h),
                                          qa, qs, out, os, lse, n, heads, ws, wsb, None)

    def move(c=None, q=None, path=buf, stride=4, n=0):
        return L.splitzip_cache_move(C.byref(cache() if c is None else c), 1, C.byref(seqs() if q is None else q), path, stride, n, None)

    bad = [(cache(dtype=3), -1), (cache(heads=0), -1), (cache(dim=96), -2), (cache(page=4), -1), (cache(pages=0), -1), (cache(res=1), -1),
           (cache(ps=8), -1), (cache(ts=1032), -1), (cache(hs=64), -1), (cache(ts=112), -1), (cache(ss=4), -1), (cache(k=None), -1), (cache(v=buf + 8), -1),
           (cache(ks=None), -1), (cache(vs=buf + 4), -1), (cache(page=24), -1)]
    for f in (write, attention, move):
        assert f() == 0                                                # no rows: nothing is launched
        for c, rc in bad:
            assert f(c=c) == rc
        for q in (seqs(starts=None), seqs(lens=None), seqs(lens=buf + 2), seqs(stride=0), seqs(table=buf + 1), seqs(table=None, n=5)):
            assert f(q=q) == -1
        assert f(q=seqs(n=1 << 16)) == -2
        assert f(q=seqs(n=0, starts=None, lens=None)) == 0
    assert write(c=cache(page=24), q=seqs(table=None, n=4)) == 0        # without a table a page is a sequence's room
    assert write(c=cache(page=20), q=seqs(table=None, n=4)) == -1
    assert write(c=cache(dtype=sz.BF16, ts=4096, hs=256, ks=None, vs=None, ss=3)) == 0
    for k in (dict(k=None), dict(v=None), dict(k=buf + 2), dict(ks=1020), dict(vs=1028)):
        assert write(n=1, **k) == -1
    assert write(n=(1 << 30) + 1) == -2
    for h in (how(cap=-1.0), how(cap=float("nan")), how(tree=buf), how(tree=buf + 4, words=1), how(slopes=buf + 2), how(pos=buf + 1), how(res=1)):
        assert attention(h=h) == -1
    assert attention(heads=12) == -1 and attention(heads=0) == -1
    for k in (dict(qa=None), dict(out=None), dict(qs=4095), dict(qs=4088), dict(os=4092), dict(qa=buf + 8), dict(lse=buf + 2)):
        assert attention(n=1, **k) == -1
    long = seqs(len=1 << 20, stride=1 << 16)
    need = L.splitzip_attention_workspace_bytes(C.byref(cache()), C.byref(long), 2, 32)
    assert need > 0 and need % 4 == 0
    assert attention(q=long, n=2, wsb=0) == -3
    assert attention(q=long, n=2, ws=None) == -1 and attention(q=long, n=2, ws=buf + 4) == -1
    assert L.splitzip_attention_workspace_bytes(C.byref(cache()), C.byref(long), 2, 12) == 0
    assert L.splitzip_attention_workspace_bytes(None, C.byref(long), 2, 32) == 0
    assert L.splitzip_attention_workspace_bytes(C.byref(cache()), C.byref(seqs(len=200)), 2, 32) == 0     # one part: no workspace
    assert move(n=1, path=None) == -1 and move(n=1, path=buf + 2) == -1 and move(n=1, stride=0) == 0
    two = (_CCache * 2)(cache(), cache(ts=2048, hs=256))
    assert L.splitzip_cache_move(two, 2, C.byref(seqs()), buf, 4, 0, None) == -1
    assert L.splitzip_cache_move(None, 2, C.byref(seqs()), buf, 4, 1, None) == -1
    assert L.splitzip_cache_move(None, 0, None, None, 0, 1, None) == 0
    assert L.splitzip_cache_write(None, C.byref(seqs()), buf, 1024, buf, 1024, 1, None) == -1
    assert L.splitzip_cache_read(C.byref(cache()), None, buf, 1024, buf, 1024, 1, None) == -1


@pytest.mark.parametrize("window", [0, 1, 100, 700, 1000, 5000])
@pytest.mark.parametrize("n", [1, 3, 16])
def test_a_workspace_is_enough_for_every_window(n, window):
    """the bytes that are asked for without a window do for a call with one (which is refused for its query, and not for them)"""
    L, buf = sz.lib(), 1 << 16
    c = _CCache(buf, buf, buf, buf, sz.FP8_E5M2, 8, 128, 16, 4, 0, 16 * 1024, 1024, 128, 128)
    for most in (1, 255, 257, 1030, 2048, 2056, 2304, 5000, 131072):
        q = _CSeqs(buf, buf, buf, 1 << 13, n, 1, most)
        need = L.splitzip_attention_workspace_bytes(C.byref(c), C.byref(q), n, 32)
        h = _CAttention(1.0, 0.0, None, None, None, 0, window, 0)
        assert L.splitzip_cache_attention(C.byref(c), C.byref(q), C.byref(h), buf + 2, 4096, buf, 4096, None, n, 32, buf, need, None) == -1


def test_python_side_checks():
    z = lambda *s, dtype=torch.uint8: torch.zeros(*s, dtype=dtype)   # noqa: E731
    kv, scales = z(3, 16, 2, 64), z(3, 2, 16)
    sz.KvCache(kv, kv, sz.FP8_E5M2, scales, scales)
    for args in ((kv, kv, sz.BF16), (kv, kv, sz.FP8_E4M3), (kv, z(3, 16, 2, 128), sz.FP8_E5M2, scales, scales), (kv[..., ::2], kv[..., ::2], sz.FP8_E5M2, scales, scales),
                 (kv, kv, sz.FP8_E5M2, scales.transpose(1, 2), scales), (kv[0], kv[0], sz.FP8_E5M2, scales, scales)):
        with pytest.raises(ValueError):
            sz.KvCache(*args)
    i32 = lambda *s: z(*s, dtype=torch.int32)   # noqa: E731
    sz.Sequences(i32(2, 4), i32(3), i32(2), 1, 64)
    for args in ((i32(2, 4), i32(2), i32(2)), (i32(3, 4), i32(3), i32(2)), (i32(2, 4), i32(3).long(), i32(2)), (i32(2, 8)[:, ::2], i32(3), i32(2))):
        with pytest.raises(ValueError):
            sz.Sequences(*args, 1, 64)
    with pytest.raises(ValueError):
        sz.Attention(1.0, tree=z(4, 1))
    with pytest.raises(ValueError):
        sz.Attention(1.0, slopes=z(4, dtype=torch.float64))
    c, q = sz.KvCache(kv, kv, sz.FP8_E5M2, scales, scales), sz.Sequences(i32(2, 4), i32(3), i32(2), 1, 64)
    x = z(2, 2, 64, dtype=torch.bfloat16)
    for k, v in ((x[:, :1], x), (x, x[:1]), (x.transpose(0, 1), x), (x.float(), x)):
        with pytest.raises(ValueError):
            sz.cache_write(k, v, c, q)
    with pytest.raises(ValueError):
        sz.cache_attention(x, c, q, x[:1], scales, sz.Attention(1.0))
    with pytest.raises(ValueError):
        sz.cache_attention(x, c, q, x, scales, sz.Attention(1.0, slopes=z(3, dtype=torch.float32)))
    with pytest.raises(ValueError):
        sz.cache_move(sz.KvCaches([c]), q, i32(3, 4))


# ---- writing and reading -------------------------------------------------------------------------------

def special_rows(n, heads, dim, seed):
    """rows with what can go wrong: zeros, subnormals, the largest and the smallest magnitudes, infinities, NaN, ties"""
    rng = np.random.default_rng(seed)
    x = rounded(rng.standard_normal((n, heads, dim)) * np.exp2(rng.integers(-30, 30, (n, heads, 1))), sz.BF16)
    flat = x.reshape(-1, dim)
    for r in range(0, flat.shape[0], 3):
        what = r // 3 % 9
        if what == 0:
            flat[r] = 0
        elif what == 1:
            flat[r] = 2.0 ** -133 * rng.integers(-127, 128, dim)              # BF16 subnormals
        elif what == 2:
            flat[r, 3], flat[r, 5] = np.inf, -np.inf
        elif what == 3:
            flat[r, 1] = np.nan
        elif what == 4:
            flat[r] = rounded(np.sign(flat[r]) * 3.3e38, sz.BF16)
        elif what == 5:
            flat[r] = 1.75 * 2.0 ** int(rng.integers(-100, 100))              # exactly the largest word of a scale
        elif what == 6:
            flat[r] = (1.75 + 2.0 ** -7) * 2.0 ** int(rng.integers(-100, 100))    # just above it
        elif what == 7:
            flat[r] = np.exp2(rng.integers(-126, 127, dim).astype(float))     # the whole range in one row
        else:
            flat[r, :] = np.inf
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,heads,page,layout", [(128, 2, 16, "nhd"), (64, 3, 8, "hnd"), (256, 1, 32, "side"), (128, 8, 16, "flat")])
def test_write_and_read_are_exact(kind, dim, heads, page, layout):
    lens, rows = [37, 1, 0, 100, 16, 5], [37, 1, 0, 13, 0, 7]           # (7 rows of 5 tokens: the first two are nowhere)
    w = World(kind, lens, rows, heads, dim, page, layout, seed=3)
    k, v = special_rows(w.n_rows, heads, dim, 1), special_rows(w.n_rows, heads, dim, 2)
    # strided rows: K and V as parts of one tensor
    both = torch.from_numpy(np.stack([k, v], 1)).to(torch.bfloat16).cuda()
    before = w.pool.clone(), None if w.scales is None else w.scales.clone()
    sz.cache_write(both[:, 0], both[:, 1], w.cache, w.seqs)
    got = [t.view(FLOATS[kind]).double().cpu().numpy() for t in (w.cache.k, w.cache.v)]
    bytes_ = None if w.scales is None else w.scales.cpu().numpy()
    fresh = torch.zeros(w.pages, w.page, dtype=torch.bool)
    for s in range(len(lens)):
        for i in range(rows[s]):
            t = lens[s] - rows[s] + i
            if t < 0:
                continue
            p, a = w.slot(s, t)
            fresh[p, a] = True
            for which, x in enumerate((k, v)):
                row = x[w.starts[s] + i]
                if kind == sz.BF16:
                    assert np.array_equal(got[which][p, a], row, equal_nan=True)
                else:
                    y, b = quantised(row, kind)
                    assert np.array_equal(bytes_[which, p, :, a], b)
                    assert np.array_equal(got[which][p, a], y, equal_nan=True)
    # and nothing else
    now = [t.clone() for t in (w.cache.k, w.cache.v)]
    w.pool.copy_(before[0])
    was = [t.clone() for t in (w.cache.k, w.cache.v)]
    for a, b in zip(now, was):
        assert torch.equal(a[~fresh.cuda()], b[~fresh.cuda()])
    if w.scales is not None:
        assert torch.equal(w.scales.transpose(2, 3)[:, ~fresh.cuda()], before[1].transpose(2, 3)[:, ~fresh.cuda()])
        w.scales.copy_(before[1])
    # back: into rows that are strided too
    sz.cache_write(both[:, 0], both[:, 1], w.cache, w.seqs)
    back = torch.full((w.n_rows, 2, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    sz.cache_read(w.cache, w.seqs, back[:, 0], back[:, 1])
    back = back.double().cpu().numpy()
    for s in range(len(lens)):
        for i in range(rows[s]):
            for which, x in enumerate((k, v)):
                row = x[w.starts[s] + i]
                if lens[s] - rows[s] + i < 0:
                    want = np.zeros_like(row)
                elif kind == sz.BF16:
                    want = row
                else:
                    y, b = quantised(row, kind)
                    want = rounded(y * np.ldexp(1.0, b.astype(int) - 127)[:, None], sz.BF16)
                assert np.array_equal(back[w.starts[s] + i, which], want, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [sz.FP8_E5M2, sz.FP8_E4M3])
def test_read_every_word_under_every_scale(kind):
    """all 256 words times all scale bytes 0 .. 254 are rounded to BF16 once"""
    words = torch.arange(256, dtype=torch.uint8).repeat(256)[: 255 * 256].view(1, 255, 256)
    k = torch.zeros(1, 256, 1, 256, dtype=torch.uint8)
    k[0, :255, 0] = words[0]
    scales = torch.zeros(1, 1, 256, dtype=torch.uint8)
    scales[0, 0, :255] = torch.arange(255, dtype=torch.uint8)
    c = sz.KvCache(k.cuda(), k.cuda(), kind, scales.cuda(), scales.cuda())
    q = sz.Sequences(None, torch.tensor([0, 255], dtype=torch.int32, device="cuda"), torch.tensor([255], dtype=torch.int32, device="cuda"), 255, 255)
    out = [torch.zeros(255, 1, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sz.cache_read(c, q, *out)
    value = k[0, :255, 0].view(FLOATS[kind]).double().numpy() * np.ldexp(1.0, np.arange(255) - 127)[:, None]
    want = rounded(value, sz.BF16)
    for o in out:
        assert np.array_equal(o[:, 0].double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.gpu
def test_launch_hints_do_not_change_what_is_written():
    """max_rows and max_len are hints: too small ones take longer, no more"""
    for hint in (0, 1, 5000):
        w = World(sz.FP8_E5M2, [900, 3], [900, 2], seed=1, max_rows=hint, max_len=hint)
        x = torch.randn(2, w.n_rows, 2, 128, device="cuda").to(torch.bfloat16)
        sz.cache_write(x[0], x[1], w.cache, w.seqs)
        y = torch.zeros_like(x)
        sz.cache_read(w.cache, w.seqs, y[0], y[1])
        assert ((y.float() - x.float()).abs() <= x.float().abs() / 8 + x.float().abs().amax(-1, keepdim=True) * 2.0 ** -15).all()   # 2 bits of mantissa: half a unit


# ---- attention -----------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,T", [(1, 1), (4, 1), (5, 3), (16, 1), (8, 3), (3, 21), (4, 33)])
def test_chains(kind, dim, group, T):
    """single tokens, drafts and pieces of prompts: every number of rows per wave, ragged lengths, empty sequences"""
    lens = [T, T + 1, 40 + T, 129, 0, 300 + T, 31 + T]
    rows = [T, T, T, T, 0, max(T - 1, 1), T]
    w = World(kind, lens, rows, 2, dim, 16, seed=T)
    q, qd = queries(w, group)
    out, lse = run(w, qd, sz.Attention(dim ** -0.5))
    close(out, lse, attend(w, q, dim ** -0.5))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page,layout", [(8, "nhd"), (16, "hnd"), (64, "side"), (128, "nhd"), (16, "flat")])
def test_layouts(kind, page, layout):
    w = World(kind, [1, 7, 8, 9, 63, 64, 65, 200], [1] * 8, 3, 128, page, layout, seed=7)
    q, qd = queries(w, 2)
    out, lse = run(w, qd, sz.Attention(0.1))
    close(out, lse, attend(w, q, 0.1))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,words", [(13, 1), (64, 1), (70, 2), (130, 3)])
def test_trees(kind, T, words):
    """a random tree per sequence, positions by depth; rows of more than 64 tokens take several words"""
    rng = np.random.default_rng(T)
    lens, rows = [T, T + 77, 300 + T], [T, T - 3, T]
    w = World(kind, lens, rows, 1, 128, 16, seed=2)
    bits, pos, sees = [], [], []
    for n, r in zip(lens, rows):
        b, d, s = random_tree(r, rng, words)
        bits.append(b)
        pos += [n - r + x for x in d]
        sees.append(s)
    q, qd = queries(w, 4)
    slopes = np.array([0.5, 0.25, 0.125, 0.0625])
    how = sz.Attention(0.09, slopes=torch.tensor(slopes, dtype=torch.float32, device="cuda"), tree=torch.from_numpy(np.concatenate(bits)).cuda(),
                       positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    out, lse = run(w, qd, how)
    close(out, lse, attend(w, q, 0.09, slopes=slopes, see=lambda s, i, j: sees[s][i] >> j & 1, positions=pos))


@pytest.mark.gpu
def test_rows_that_see_nothing():
    """a tree mask of zeros over no cached tokens; bits that the words do not reach; a window of nothing but the future"""
    w = World(sz.BF16, [5, 9, 70], [5, 5, 70], 2, 64, 8, seed=4)
    tree = torch.zeros(80, 1, dtype=torch.int64, device="cuda")
    tree[2] = 0b10100
    tree[79] = -1
    sees = lambda s, i, j: (s == 0 and i == 2 and j in (2, 4)) or (s == 2 and i == 69 and j < 64)   # noqa: E731
    q, qd = queries(w, 2)
    out, lse = run(w, qd, sz.Attention(0.1, tree=tree))
    want = attend(w, q, 0.1, see=sees)
    assert np.isneginf(want[1][0]).all() and np.isfinite(want[1][5]).all()
    close(out, lse, want)
    assert (out[0] == 0).all() and (out[78] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("softcap,window,bias,T", [(30.0, 0, False, 1), (0.0, 50, False, 1), (5.0, 33, True, 4), (0.0, 1, False, 3), (20.0, 0, True, 40),
                                                   (0.0, 1 << 31, True, 2)])
def test_capped_windowed_biased(kind, softcap, window, bias, T):
    lens = [T, 64 + T, 257, 1500]
    w = World(kind, lens, [T] * 4, 2, 128, 32, seed=9)
    q, qd = queries(w, 3)
    q, qd = q * 4, qd * 4
    slopes = 2.0 ** -np.arange(1, 7) if bias else None
    how = sz.Attention(0.088, softcap=softcap, window=window, slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda"))
    out, lse = run(w, qd, how)
    close(out, lse, attend(w, q, 0.088, softcap=softcap, window=window, slopes=slopes))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [sz.BF16, sz.FP8_E4M3])
def test_long_sequences_in_parts(kind):
    """parts, their join, and hints that are too small: the last part and the last tile of rows go on to the end"""
    w = World(kind, [3001, 1, 2000, 700], [2, 1, 9, 9], 1, 128, 16, seed=11)
    q, qd = queries(w, 4)
    want = attend(w, q, 0.1)
    close(*run(w, qd, sz.Attention(0.1)), want)
    for rows, most in ((1, 3001), (9, 300), (0, 0), (100, 100000)):
        w.seqs = sz.Sequences(*w.dev, max_rows=rows, max_len=most)
        close(*run(w, qd, sz.Attention(0.1)), want)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 7, 40])
def test_many_sequences(rows):
    """more than 64 sequences: their blocks are summed up 64 at a time, and a workgroup takes several of them"""
    rng = np.random.default_rng(rows)
    lens = [int(x) for x in rng.integers(0, 90, 150)] + [900, 0, 500]
    T = [min(rows, n) if k % 5 else 0 for k, n in enumerate(lens)]
    w = World(sz.FP8_E5M2, lens, T, 1, 64, 16, seed=rows)
    q, qd = queries(w, 2)
    want = attend(w, q, 0.1)
    close(*run(w, qd, sz.Attention(0.1)), want)
    w.seqs = sz.Sequences(*w.dev, max_rows=rows, max_len=60)          # cut for short sequences: every one as a whole
    close(*run(w, qd, sz.Attention(0.1)), want)


@pytest.mark.gpu
def test_the_short_way_and_the_general_way(monkeypatch):
    """what lib().fast_cache takes gives the bits that the ctypes calls give, and what it does not take is refused or taken by them"""
    w = World(sz.FP8_E4M3, [300, 70], [3, 3], 2, 128, 16, seed=30)
    q, qd = queries(w, 4)
    path = torch.tensor([[0, 2], [1, -1]], dtype=torch.int32, device="cuda")
    new = torch.randn(2, w.n_rows, 2, 128, device="cuda").to(torch.bfloat16)
    tree = torch.tensor([1, 3, 7, 1, 2, 4], device="cuda")[:, None].contiguous()

    def all_calls():
        sz.cache_write(new[0], new[1], w.cache, w.seqs)
        out, lse = run(w, qd, sz.Attention(0.1, tree=tree))
        back = torch.zeros_like(new)
        sz.cache_read(w.cache, w.seqs, back[0], back[1])
        sz.cache_move(sz.KvCaches([w.cache]), w.seqs, path)
        return out, lse, back, w.cache.k.clone(), w.scales.clone()

    L, before, scales = sz.lib(), w.pool.clone(), w.scales.clone()
    taken = []
    for name in ("splitzip_cache_write", "splitzip_cache_read", "splitzip_cache_attention", "splitzip_cache_move"):
        f = getattr(L.fast_cache, name)
        monkeypatch.setattr(L.fast_cache, name, lambda *a, f=f: taken.append(f(*a)) or taken[-1])
    first = all_calls()
    assert taken == [0, 0, 0, 0]
    for name in ("splitzip_cache_write", "splitzip_cache_read", "splitzip_cache_attention", "splitzip_cache_move"):
        monkeypatch.setattr(L.fast_cache, name, lambda *a: 1)
    w.pool.copy_(before)
    w.scales.copy_(scales)
    for a, b in zip(first, all_calls()):
        assert torch.equal(a, b)


def test_other_forms_are_left_to_the_general_way():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)   # noqa: E731
    c, q = sz.KvCache(z(3, 16, 2, 64), z(3, 16, 2, 64), sz.BF16), sz.Sequences(z(2, 4, dtype=torch.int32), z(3, dtype=torch.int32), z(2, dtype=torch.int32), 1, 64)
    f, x, how = sz.lib().fast_cache, z(2, 2, 64), sz.Attention(1.0)
    assert f.splitzip_cache_write(c.c, q.c, x, x, 0) == 1                 # tensors in host memory
    assert f.splitzip_cache_write(q.c, c.c, x, x, 0) == 1                 # another structure
    assert f.splitzip_cache_attention(c.c, q.c, how.c, x, x, None, x, None, 0) == 1
    assert f.splitzip_cache_attention(c.c, q.c, _CAttention(), x, x, None, x, None, 0) == 1
    assert f.splitzip_cache_move(sz.KvCaches([c]).items, 1, q.c, x, 1, 0) == 1


@pytest.mark.gpu
def test_positions_that_are_far_from_the_slots():
    """positions are the caller's: far below the slots they lie in, or above, with a window that then sees much or nothing"""
    w = World(sz.BF16, [1200, 1200, 1200], [3, 3, 3], 1, 64, 16, seed=12)
    q, qd = queries(w, 2)
    pos = [100, 90, 1500, 5000, 5001, 5000, -50, -51, -52]
    how = sz.Attention(0.1, window=64, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    close(*run(w, qd, how), attend(w, q, 0.1, window=64, positions=pos))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 40])
def test_what_a_row_does_not_see_does_not_touch_it(T):
    """infinities and NaN in drafted tokens off a row's path, and behind its window; those that it sees reach it"""
    w = World(sz.BF16, [100 + T, 60 + T], [T, T], 1, 128, 16, seed=13)
    q, qd = queries(w, 2)
    clean = attend(w, q, 0.1)
    w.set(0, 100 + T - 1, 0, 0, np.full(128, np.nan))      # K of the last row
    w.set(0, 100 + T - 1, 1, 0, np.full(128, np.inf))      # and V
    w.set(1, 60 + T - 1, 1, 0, np.where(np.arange(128) == 77, -np.inf, 1.0))
    out, lse = run(w, qd, sz.Attention(0.1))
    rows = np.ones(2 * T, bool)
    rows[[T - 1, 2 * T - 1]] = False
    close(out[torch.from_numpy(rows)], lse[torch.from_numpy(rows)], tuple(x[rows] for x in clean))
    got = out.double().cpu().numpy()
    assert np.isnan(got[T - 1]).all()
    assert np.isneginf(got[2 * T - 1, :, 77]).all() and np.isfinite(np.delete(got[2 * T - 1], 77, 1)).all()
    # behind the window
    w = World(sz.BF16, [200 + T], [T], 1, 128, 16, seed=14)
    q, qd = queries(w, 2)
    for t in (0, 150, 165, 200 + T - 38):
        w.set(0, t, 0, 0, np.full(128, np.inf))
        w.set(0, t, 1, 0, np.full(128, np.nan))
    out, lse = run(w, qd, sz.Attention(0.1, window=36))
    rows = np.array([not any(0 <= 200 + i - t < 36 for t in (0, 150, 165, 200 + T - 38)) for i in range(T)])
    assert rows[-1]
    for t in (0, 150, 165, 200 + T - 38):
        p, a = w.slot(0, t)
        w.value[:, p, a] = 0    # (the oracle never takes them for these rows)
    want = attend(w, q, 0.1, window=36)
    close(out[torch.from_numpy(rows)], lse[torch.from_numpy(rows)], tuple(x[rows] for x in want))
    assert torch.isnan(out[torch.from_numpy(~rows)]).all() or not (~rows).any()


@pytest.mark.gpu
def test_extreme_scores():
    """scores of hundreds, a NaN in a query, and all scores minus infinity"""
    w = World(sz.BF16, [300, 40, 33], [1, 1, 1], 1, 64, 16, seed=15)
    q, qd = queries(w, 1)
    big, bigd = rounded(q * 60, sz.BF16), torch.from_numpy(rounded(q * 60, sz.BF16)).to(torch.bfloat16).cuda()
    want = attend(w, big, 1.0)
    assert want[1].max() > 300
    close(*run(w, bigd, sz.Attention(1.0)), want)
    bigd[1, 0, 5] = float("nan")
    out, lse = run(w, bigd, sz.Attention(1.0))
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all() and torch.isfinite(out[[0, 2]]).all()
    for t in range(33):
        w.set(2, t, 0, 0, np.where(np.arange(64) == 0, -np.inf, 0.0))
    qd[2] = 1.0
    out, lse = run(w, qd, sz.Attention(1.0))
    assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()


@pytest.mark.gpu
def test_strided_rows_other_streams_graphs_and_repeats():
    """rows inside a wider tensor; a stream of the caller's; a captured call replayed with other lengths; the same bits every time"""
    w = World(sz.FP8_E5M2, [2000, 400, 33], [2, 2, 2], 2, 128, 16, seed=16)
    q, qd = queries(w, 4)
    wide = torch.full((w.n_rows, 8, 3 * 128), 9.0, dtype=torch.bfloat16, device="cuda").view(w.n_rows, 3, 8, 128)
    wide[:, 1] = qd
    how = sz.Attention(0.1)
    first, lse1 = run(w, wide[:, 1], how, out=wide[:, 2])
    close(first, lse1, attend(w, q, 0.1))
    assert (wide[:, 0] == 9).all()
    out, lse = torch.zeros_like(qd), torch.zeros(qd.shape[:2], device="cuda")
    ws = sz.attention_workspace(w.cache, w.seqs, w.n_rows, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sz.cache_attention(qd, w.cache, w.seqs, out, ws, how, lse, stream=side)
    side.synchronize()
    assert torch.equal(out, first) and torch.equal(lse, lse1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sz.cache_attention(qd, w.cache, w.seqs, out, ws, how, lse)
    for lens in ([2000, 400, 33], [1500, 2, 20], [5, 400, 33], [2000, 400, 33]):
        w.dev[2].copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        w.lens = lens
        close(out, lse, attend(w, q, 0.1))
    assert torch.equal(out, first)


@pytest.mark.gpu
def test_what_device_memory_says_leads_nowhere_outside():
    """lengths, starts and table entries beyond the buffers are clamped (results undefined, no access outside)"""
    w = World(sz.BF16, [40, 50], [2, 2], 1, 64, 16, seed=17)
    q, qd = queries(w, 2)
    for lens, starts, table in (([1 << 30, -5], [0, 2, 4], None), ([40, 50], [-3, 2, 1 << 20], None), ([40, 50], [3, 1, 4], None), ([40, 50], [0, 2, 4], -1)):
        w.dev[2].copy_(torch.tensor(lens, dtype=torch.int32))
        w.dev[1].copy_(torch.tensor(starts, dtype=torch.int32))
        if table is not None:
            w.dev[0].fill_(table)
        run(w, qd, sz.Attention(0.1))
        x = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
        sz.cache_write(x, x, w.cache, w.seqs)
        sz.cache_read(w.cache, w.seqs, x, x)
        sz.cache_move(sz.KvCaches([w.cache]), w.seqs, torch.tensor([[0, 1, 7], [1, 0, -1]], dtype=torch.int32, device="cuda"), n_rows=4)
    torch.cuda.synchronize()


# ---- moving an accepted path ---------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layers,layout", [(1, "nhd"), (3, "side"), (66, "nhd")])
def test_move(kind, layers, layout):
    lens, rows = [64, 13, 40, 9, 7, 90], [13, 13, 20, 9, 9, 30]      # (nine rows of seven tokens: the first two are nowhere)
    paths = [[0, 2, 5, 9, 12, -1], [1, 3, 4, 11, -1, -1], [0, 1, 2, 3, 4, 19], [-1, 3, 4, -1, -1, -1], [3, 4, 6, 8, -1, -1], [5, 8, 7, 20, 29, 30]]
    valid = [[0, 2, 5, 9, 12], [1, 3, 4, 11], [0, 1, 2, 3, 4, 19], [], [3, 4, 6, 8], [5, 8]]
    worlds = [World(kind, lens, rows, 2, 64, 8, layout, seed=20, junk=False) for _ in range(min(layers, 3))]
    # layers of one geometry and one table, their words told apart
    caches, tensors = [], []
    for layer in range(layers):
        w = worlds[0]
        pool = torch.randint(0, 256, w.pool.shape, dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(layer)).to(w.pool.dtype)
        scales = None if w.scales is None else torch.randint(0, 200, w.scales.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(layer)).to(torch.uint8)
        k, v = (pool[:, 0], pool[:, 1]) if layout == "side" else (pool[0], pool[1])
        caches.append(sz.KvCache(k, v, kind, *([None, None] if scales is None else scales)))
        tensors.append((k, v, scales))
    want = [(k.cpu().clone(), v.cpu().clone(), None if b is None else b.cpu().clone()) for k, v, b in tensors]
    w = worlds[0]
    for (k, v, b), (k0, v0, b0) in zip(want, [(k.cpu(), v.cpu(), None if b is None else b.cpu()) for k, v, b in tensors]):
        for s, path in enumerate(valid):
            base = lens[s] - rows[s]
            for i, a in enumerate(path):
                if base + i < 0:
                    continue
                (p0, t0), (p1, t1) = w.slot(s, base + a), w.slot(s, base + i)
                k[p1, t1], v[p1, t1] = k0[p0, t0], v0[p0, t0]
                if b is not None:
                    b[:, p1, :, t1] = b0[:, p0, :, t0]
    sz.cache_move(sz.KvCaches(caches), w.seqs, torch.tensor(paths, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for (k, v, b), (k1, v1, b1) in zip(tensors, want):
        assert torch.equal(k.cpu(), k1) and torch.equal(v.cpu(), v1)
        assert b is None or torch.equal(b.cpu(), b1)


@pytest.mark.gpu
def test_a_step_with_drafts_and_the_way_of_the_cache():
    """write, attention, move, compress, decompress and read as a program uses them (paper_2605_01708_amd.tree_decode)"""
    from paper_2605_01708_amd import tree_decode

    outs, lens, ratio, same = tree_decode.step(tokens=300, sequences=3, layers=2, drafts=13)
    assert same and ratio > 1.0
    assert lens == [303, 266, 229]
    assert all(torch.isfinite(o).all() and o.shape == (39, 32, 128) for o in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dim", [(sz.BF16, 128), (sz.FP8_E5M2, 64), (sz.FP8_E4M3, 256)])
@pytest.mark.parametrize("window", [0, 100])
def test_pieces_of_prompts(kind, dim, window):
    """several tiles of rows, each of which sees another length; over nothing, over a prefix, and more rows than tokens"""
    w = World(kind, [200, 777, 60, 150], [200, 180, 60, 170], 1, dim, 16, seed=dim, max_len=777)
    q, qd = queries(w, 3)
    want = attend(w, q, 0.1, window=window)
    close(*run(w, qd, sz.Attention(0.1, window=window)), want)
    w.seqs = sz.Sequences(*w.dev, max_rows=16, max_len=100)
    close(*run(w, qd, sz.Attention(0.1, window=window)), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,T", [(64, 64), (128, 64), (128, 16), (256, 5)])
def test_parts_of_trees(dim, T):
    """one long sequence in many parts, in every kernel: a random tree at its end"""
    rng = np.random.default_rng(dim + T)
    w = World(sz.FP8_E5M2, [T + 2500], [T], 1, dim, 16, seed=3)
    bits, depth, sees = random_tree(T, rng, 1)
    q, qd = queries(w, 6)
    pos = [2500 + d for d in depth]
    how = sz.Attention(0.08, window=2400, tree=torch.from_numpy(bits).cuda(), positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    want = attend(w, q, 0.08, window=2400, see=lambda s, i, j: sees[i] >> j & 1, positions=pos)
    first = run(w, qd, how)
    close(*first, want)
    for a, b in zip(first, run(w, qd, how)):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 30])
@pytest.mark.parametrize("scale,softcap", [(-0.1, 0.0), (0.0, 0.0), (-0.1, 7.0), (0.1, 5000.0), (0.1, 1e30), (0.3, 1e-20)])
def test_scales_and_caps(T, scale, softcap):
    """scales of either sign and none; a cap so wide that it does nothing costs no precision, and one that leaves nothing is no NaN"""
    w = World(sz.BF16, [300, 40], [T, T], 2, 128, 16, seed=17)
    q, qd = queries(w, 2)
    out, lse = run(w, qd, sz.Attention(scale, softcap=softcap))
    want = list(attend(w, q, scale, softcap=softcap if softcap < 1000 else 0.0))
    x = abs(scale) * 4 * 128                                              # more than any score here
    want[3] = np.abs(attend(w, q, abs(scale))[3]) + 4e-7 * min(softcap, x) + (x ** 3 / softcap ** 2 / 3 if softcap >= 1000 else 0.0)
    close(out, lse, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 40])
def test_what_all_rows_see_reaches_them(T):
    """an infinity that every row sees, in 32 tokens of which some rows see a part only, and one in front of them"""
    w = World(sz.BF16, [100 + T, 400 + T], [T, T], 1, 128, 16, seed=19)
    q, qd = queries(w, 2)
    w.set(0, 99, 1, 0, np.where(np.arange(128) == 3, np.inf, 1.0))
    w.set(0, 100, 1, 0, np.where(np.arange(128) == 70, -np.inf, 1.0))
    w.set(1, 20, 1, 0, np.where(np.arange(128) == 127, np.nan, 1.0))
    out = run(w, qd, sz.Attention(0.1))[0].double().cpu().numpy()
    assert np.isposinf(out[:T, :, 3]).all() and np.isneginf(out[:T, :, 70]).all() and np.isnan(out[T:, :, 127]).all()
    assert np.isfinite(np.delete(out[:T], [3, 70], 2)).all() and np.isfinite(np.delete(out[T:], 127, 2)).all()


@pytest.mark.gpu
def test_a_pool_beyond_32_bits():
    """pages more than 4 GiB from the pool's start: written, read, moved and attended to there"""
    pages = (5 << 30) // (16 * 1024)
    k, v = (torch.empty(pages, 16, 8, 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    scales = torch.zeros(2, pages, 8, 16, dtype=torch.uint8, device="cuda")
    far = sz.KvCache(k, v, sz.FP8_E4M3, scales[0], scales[1])
    near = sz.KvCache.zeros(8, 16, 8, 128, sz.FP8_E4M3)
    x = torch.randn(2, 100, 8, 128, device="cuda").to(torch.bfloat16)
    q = torch.randn(4, 8, 128, device="cuda").to(torch.bfloat16)
    got = []
    for cache, first in ((far, pages - 8), (near, 0)):
        table = torch.arange(first, first + 8, dtype=torch.int32, device="cuda")[None].contiguous()
        i32 = lambda *y: torch.tensor(y, dtype=torch.int32, device="cuda")   # noqa: E731
        sz.cache_write(x[0], x[1], cache, sz.Sequences(table, i32(0, 100), i32(100), 100, 100))
        step = sz.Sequences(table, i32(0, 4), i32(100), 4, 100)
        sz.cache_move(sz.KvCaches([cache]), step, i32(0, 2, 3)[None].contiguous())
        back, out = torch.zeros_like(x), torch.zeros_like(q)
        sz.cache_read(cache, sz.Sequences(table, i32(0, 100), i32(100), 100, 100), back[0], back[1])
        sz.cache_attention(q, cache, step, out, sz.attention_workspace(cache, step, 4, 8), sz.Attention(0.1))
        got += [back, out]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3]) and got[0].abs().sum() > 0


def test_strides_and_caps_beyond_the_limits_are_refused():
    L, buf = sz.lib(), 1 << 16

    def need(**k):
        d = dict(k=buf, v=buf, ks=buf, vs=buf, dtype=sz.FP8_E5M2, heads=8, dim=128, page=16, pages=4, res=0, ps=16 * 1024, ts=1024, hs=128, ss=128)
        d.update(k)
        c = _CCache(*[d[x] for x in ("k", "v", "ks", "vs", "dtype", "heads", "dim", "page", "pages", "res", "ps", "ts", "hs", "ss")])
        return L.splitzip_cache_write(c, _CSeqs(buf, buf, buf, 4, 0, 1, 64), buf, 1024, buf, 1024, 0, None)

    assert need() == 0
    assert need(ts=1 << 28) == 0 and need(ts=(1 << 28) + 16) == -2
    assert need(ps=(1 << 32) - 16) == 0 and need(ps=1 << 32) == -2
    assert need(ss=(1 << 32) - 8) == 0 and need(ss=1 << 32) == -2
    c = _CCache(buf, buf, buf, buf, sz.FP8_E5M2, 8, 128, 16, 4, 0, 16 * 1024, 1024, 128, 128)
    for cap, rc in ((0.0, 0), (30.0, 0), (-1.0, -1), (math.nan, -1), (math.inf, -1), (1e-40, -1)):
        how = _CAttention(1.0, cap, None, None, None, 0, 0, 0)
        assert L.splitzip_cache_attention(c, _CSeqs(buf, buf, buf, 4, 0, 1, 64), how, buf, 1024, buf, 1024, None, 0, 8, None, 0, None) == rc
