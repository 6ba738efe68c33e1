"""What the binding's cache calls refuse before an address reaches the GPU: tensors in host memory and of other types.

The calls here have no rows, so that nothing is launched whatever they say."""
import ctypes as C

import pytest
import torch

import paper_2605_01708_amd as sz
from paper_2605_01708_amd.binding import _CAttention, _CCache, _CSeqs

I32 = torch.int32


def world(device, where=()):
    """descriptions and tensors of a call without rows, on the device but for those named in `where`, which are in host memory"""
    def z(name, *shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device="cpu" if name in where else device)

    u8 = torch.uint8
    cache = sz.KvCache(z("k", 3, 16, 2, 64, dtype=u8), z("v", 3, 16, 2, 64, dtype=u8), sz.FP8_E5M2, z("k_scales", 3, 2, 16, dtype=u8), z("v_scales", 3, 2, 16, dtype=u8))
    seqs = sz.Sequences(z("table", 2, 4, dtype=I32), z("starts", 3, dtype=I32), z("lens", 2, dtype=I32), 1, 64)
    how = sz.Attention(1.0, slopes=z("slopes", 4, dtype=torch.float32), tree=z("tree", 0, 1, dtype=torch.int64), positions=z("positions", 0, dtype=I32))
    rows = {name: z(name, 0, 2, 64) for name in ("new_k", "new_v")}
    rows |= {name: z(name, 0, 4, 64) for name in ("q", "out")}
    return cache, seqs, how, {**rows, "lse": z("lse", 0, 4, dtype=torch.float32), "workspace": z("workspace", 64, dtype=u8), "path": z("path", 2, 3, dtype=I32)}


def calls(cache, seqs, how, t):
    return {"write": lambda: sz.cache_write(t["new_k"], t["new_v"], cache, seqs), "read": lambda: sz.cache_read(cache, seqs, t["new_k"], t["new_v"]),
            "attention": lambda: sz.cache_attention(t["q"], cache, seqs, t["out"], t["workspace"], how, t["lse"]),
            "move": lambda: sz.cache_move(sz.KvCaches([cache]), seqs, t["path"], n_rows=0)}


SHARED = ("k", "v", "k_scales", "v_scales", "table", "starts", "lens")
OWN = {"write": ("new_k", "new_v"), "read": ("new_k", "new_v"), "attention": ("slopes", "tree", "positions", "q", "out", "lse", "workspace"), "move": ("path",)}


@pytest.mark.parametrize("name", OWN)
def test_host_memory_is_refused(name):
    with pytest.raises(ValueError, match="on the GPU"):
        calls(*world("cpu"))[name]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", OWN)
def test_a_single_tensor_in_host_memory_is_refused(name):
    calls(*world("cuda"))[name]()
    for what in SHARED + OWN[name]:
        with pytest.raises(ValueError, match="on the GPU"):
            calls(*world("cuda", (what,)))[name]()


@pytest.mark.gpu
def test_a_workspace_of_repeated_bytes_is_refused():
    cache, seqs, how, t = world("cuda")
    t["workspace"] = torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 20)
    with pytest.raises(ValueError, match="contiguous"):
        calls(cache, seqs, how, t)["attention"]()


@pytest.mark.gpu
def test_pinned_memory_is_reached():
    """what the GPU reaches is taken: a table, starts and lengths in pinned host memory"""
    i32 = lambda *x: torch.tensor(x, dtype=I32)   # noqa: E731
    cache = sz.KvCache.zeros(4, 16, 2, 64, sz.BF16)
    x = torch.randn(2, 21, 2, 64, device="cuda").to(torch.bfloat16)
    seqs = sz.Sequences(i32(2, 1)[None].pin_memory(), i32(0, 21).pin_memory(), i32(21).pin_memory(), 21, 21)
    sz.cache_write(x[0], x[1], cache, seqs)
    y = torch.zeros_like(x)
    sz.cache_read(cache, seqs, y[0], y[1])
    torch.cuda.synchronize()
    assert torch.equal(x, y) and torch.equal(cache.k[2], x[0, :16])


# ---- types: the calls compute with the words, so that others of the same size are no words of theirs -----

@pytest.mark.parametrize("dtype,wrong", [(sz.BF16, (torch.float16,)), (sz.FP8_E5M2, (torch.float8_e4m3fn, torch.float8_e5m2fnuz, torch.bool)),
                                         (sz.FP8_E4M3, (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.bool))])
def test_words_of_another_type_are_no_cache(dtype, wrong):
    right = {sz.BF16: (torch.bfloat16, torch.int16, torch.uint16), sz.FP8_E5M2: (torch.float8_e5m2, torch.uint8, torch.int8),
             sz.FP8_E4M3: (torch.float8_e4m3fn, torch.uint8, torch.int8)}[dtype]
    scales = torch.zeros(3, 2, 16, dtype=torch.uint8)
    of = lambda t: torch.zeros(3, 16, 2, 64, dtype=torch.uint8 if t.itemsize == 1 else torch.int16).view(t)   # noqa: E731
    for t in right:
        sz.KvCache(of(t), of(t), dtype, scales, scales)
    for t in wrong:
        for k, v in ((t, right[0]), (right[0], t)):
            with pytest.raises(ValueError, match="words of the dtype"):
                sz.KvCache(of(k), of(v), dtype, scales, scales)


def refused_as_rows(device, right, wrong):
    cache, seqs, how, t = world(device)
    for name, tensors in (("write", ("new_k", "new_v")), ("read", ("new_k", "new_v")), ("attention", ("q", "out"))):
        for dtype in right:
            calls(cache, seqs, how, {**t, **{x: t[x].view(dtype) for x in tensors}})[name]()
        for x in tensors:
            for dtype in wrong:
                with pytest.raises(ValueError, match="bfloat16"):
                    calls(cache, seqs, how, {**t, x: t[x].to(dtype)})[name]()


def test_rows_of_another_type_are_refused_by_the_general_way():
    refused_as_rows("cpu", (), (torch.float16, torch.float32, torch.uint8))


@pytest.mark.gpu
def test_rows_of_another_type_are_refused():
    refused_as_rows("cuda", (torch.int16, torch.uint16), (torch.float16, torch.float32, torch.uint8))


def test_numbers_of_another_type_are_refused():
    """tables, lengths, starts, positions, paths and masks are whole numbers; 32 or 64 bits of another type are none of them"""
    i32, f32 = torch.zeros(2, 4, dtype=I32), torch.zeros(2, 4)
    starts, lens = torch.zeros(3, dtype=I32), torch.zeros(2, dtype=I32)
    for args in ((f32, starts, lens), (i32, starts.float(), lens), (i32, starts, lens.float())):
        with pytest.raises(ValueError, match="32-bit"):
            sz.Sequences(*args, 1, 64)
    for how in (dict(tree=torch.zeros(2, 1, dtype=torch.float64)), dict(tree=torch.zeros(2, 1, dtype=torch.complex64)), dict(positions=torch.zeros(2))):
        with pytest.raises(ValueError, match="integers|64-bit words"):
            sz.Attention(1.0, **how)
    kv = torch.zeros(3, 16, 2, 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="scales"):
        sz.KvCache(kv, kv, sz.FP8_E5M2, *[torch.zeros(3, 2, 16, dtype=torch.uint8).view(torch.float8_e4m3fn)] * 2)
    sz.KvCache(kv, kv, sz.FP8_E5M2, *[torch.zeros(3, 2, 16, dtype=torch.uint8).view(torch.float8_e8m0fnu)] * 2)
    sz.Sequences(i32.view(torch.uint32), starts, lens.view(torch.uint32), 1, 64)
    sz.Attention(1.0, tree=torch.zeros(2, 1, dtype=torch.uint64), positions=torch.zeros(2, dtype=I32))


def path_of_floats(device):
    cache, seqs, how, t = world(device)
    with pytest.raises(ValueError, match="32-bit integers"):
        calls(cache, seqs, how, {**t, "path": t["path"].float()})["move"]()


def test_a_path_of_floats_is_refused_by_the_general_way():
    path_of_floats("cpu")


@pytest.mark.gpu
def test_a_path_of_floats_is_refused():
    path_of_floats("cuda")


@pytest.mark.parametrize("heads,rc", [((1 << 24) - 1, -1), (1 << 24, -1), ((1 << 24) + 1, -2), (1 << 25, -2)])
def test_rows_that_offsets_of_32_bits_do_not_span_are_refused(heads, rc):
    """(the calls have no tensors, which is what rows of up to 2^31 bytes are refused for)"""
    L, buf = sz.lib(), 1 << 16
    c = _CCache(buf, buf, buf, buf, sz.FP8_E5M2, heads, 64, 8, 1, 0, 8 * 64, 64, 8 * 64, 8 * heads)
    q = _CSeqs(buf, buf, buf, 1, 1, 1, 8)
    for f in (L.splitzip_cache_write, L.splitzip_cache_read):
        assert f(C.byref(c), C.byref(q), None, 64 * heads, None, 64 * heads, 1, None) == rc
    how = _CAttention(1.0, 0.0, None, None, None, 0, 0, 0)
    assert L.splitzip_cache_attention(C.byref(c), C.byref(q), C.byref(how), None, 64 * heads, None, 64 * heads, None, 1, heads, None, 0, None) == rc


@pytest.mark.parametrize("args", [dict(drafts=65), dict(drafts=0), dict(tokens=111, sequences=4), dict(sequences=0), dict(layers=0)])
def test_the_example_says_what_it_takes(args):
    from paper_2605_01708_amd import tree_decode

    with pytest.raises(ValueError, match="64 drafts"):
        tree_decode.step(**args)


@pytest.mark.gpu
@pytest.mark.parametrize("args", [dict(tokens=40, sequences=2, layers=1, drafts=64), dict(tokens=1, sequences=1, layers=1, drafts=1)])
def test_the_example_takes_its_extremes(args):
    from paper_2605_01708_amd import tree_decode

    outs, lens, ratio, same = tree_decode.step(**args)
    assert same and all(torch.isfinite(o).all() for o in outs)
