"""ctypes binding of include/splitzip.h.  Same names as the C entry points
(without the ``splitzip_`` prefix); torch tensors supply device pointers and
the current HIP stream, nothing else.

The calls that a serving loop repeats go through the extension module _fastcall first, which marshals the plain form of
their arguments in one step (lib().fast and fast_cache, by the names of the C entry points) and answers _NOT_TAKEN for any other form; the
ctypes call behind it takes every form and raises the errors, and serves every call where the module is not there."""
from __future__ import annotations

import ctypes as C
import os
import types
import warnings

import torch

BF16 = 0
FP8_E5M2 = 1
FP8_E4M3 = 2   # accepted by the variant_* and the cache_* calls only
FP4_E2M1 = 16  # by the cache_* calls only
ESC_POS, ESC_SENTINEL, ESC_ABS32 = 0, 1, 2

STATUS_OVERFLOW = 1
STATUS_BAD_STREAM = 2
STATUS_INTERNAL = 4

ALLOT_PAGES, ALLOT_ROWS, ALLOT_LENGTH, ALLOT_POOL = 1, 2, 4, 8   # what a step's status may have (splitzip_allot_status)

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_HERE, "libsplitzip.so")


class SplitZipError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {lib().splitzip_strerror(code).decode()} ({code})")


class _CCodebook(C.Structure):
    _fields_ = [("dec", C.c_uint8 * 16), ("enc", C.c_uint8 * 256), ("member", C.c_uint8 * 256),
                ("dtype", C.c_uint32)]


class _CSizes(C.Structure):
    _fields_ = [("total_bytes", C.c_uint64), ("n_escapes", C.c_uint64), ("status", C.c_uint32),
                ("reserved", C.c_uint32)]


class _CItem(C.Structure):
    _fields_ = [("d_in", C.c_void_p), ("n_elems", C.c_uint64), ("d_out", C.c_void_p), ("out_capacity", C.c_size_t),
                ("cb", C.POINTER(_CCodebook))]


class _CDItem(C.Structure):
    _fields_ = [("d_comp", C.c_void_p), ("comp_bytes", C.c_size_t), ("n_elems", C.c_uint64), ("d_out", C.c_void_p),
                ("cb", C.POINTER(_CCodebook))]


class _CPaged(C.Structure):
    _fields_ = [("d_pool", C.c_void_p), ("d_block_table", C.c_void_p), ("n_blocks", C.c_uint32),
                ("n_pool_blocks", C.c_uint32), ("block_elems", C.c_uint32), ("reserved", C.c_uint32),
                ("page_stride_bytes", C.c_uint64), ("offset_bytes", C.c_uint64)]


class _CCache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_scales", C.c_void_p), ("d_v_scales", C.c_void_p),
                ("dtype", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("page_tokens", C.c_uint32),
                ("n_pages", C.c_uint32), ("reserved", C.c_uint32), ("page_stride_bytes", C.c_uint64),
                ("token_stride_bytes", C.c_uint64), ("head_stride_bytes", C.c_uint64), ("scale_page_stride_bytes", C.c_uint64)]


class _CSeqs(C.Structure):
    _fields_ = [("d_block_table", C.c_void_p), ("d_starts", C.c_void_p), ("d_lens", C.c_void_p), ("table_stride", C.c_uint32),
                ("n_seqs", C.c_uint32), ("max_rows", C.c_uint32), ("max_len", C.c_uint32)]


class _CRotation(C.Structure):
    _fields_ = [("d_freqs", C.c_void_p), ("d_q_weight", C.c_void_p), ("d_k_weight", C.c_void_p), ("d_positions", C.c_void_p),
                ("scaling", C.c_float), ("eps", C.c_float), ("weight_offset", C.c_float), ("rotary_dim", C.c_uint32),
                ("interleaved", C.c_uint32), ("norm", C.c_uint32), ("weights_f32", C.c_uint32), ("reserved", C.c_uint32)]


class _CRotationOf(_CRotation):
    """and how many elements its weights have and how many rows its positions (-1: none), which the calls compare with their tensors"""
    _fields_ = [("dim", C.c_int64), ("position_rows", C.c_int64)]


class _CPool(C.Structure):
    _fields_ = [("d_free", C.c_void_p), ("d_state", C.c_void_p), ("n_pages", C.c_uint32), ("page_tokens", C.c_uint32), ("reserved", C.c_uint64)]


class _CAttention(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("d_slopes", C.c_void_p), ("d_tree", C.c_void_p),
                ("d_positions", C.c_void_p), ("tree_words", C.c_uint32), ("window", C.c_uint32), ("reserved", C.c_uint64)]


class _CAttentionOf(_CAttention):
    """and how many entries its slopes, tree and positions have (-1: none), which the calls compare with their tensors"""
    _fields_ = [("heads", C.c_int64), ("tree_rows", C.c_int64), ("position_rows", C.c_int64)]


class _CCacheElsewhere(_CCache):
    """of tensors that the GPU does not reach: another type, which the short way does not take"""


class _CSeqsElsewhere(_CSeqs):
    """the same"""


class _CAttentionElsewhere(_CAttentionOf):
    """the same"""


class _CRotationElsewhere(_CRotationOf):
    """the same"""


class _CPoolElsewhere(_CPool):
    """the same"""


class Variant(C.Structure):
    """splitzip_variant: one of the formats of the paper's ablations"""
    _fields_ = [("dtype", C.c_uint32), ("code_bits", C.c_uint32), ("k", C.c_uint32), ("escape_mode", C.c_uint32),
                ("chunk_elems", C.c_uint32), ("value_bits", C.c_uint32)]

    def __repr__(self):
        return (f"Variant(dtype={self.dtype}, code_bits={self.code_bits}, k={self.k}, "
                f"escape_mode={self.escape_mode}, chunk_elems={self.chunk_elems}, value_bits={self.value_bits})")


_lib = None


def lib():
    """The loaded C library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build it with `python -m paper_2605_01708_amd.build` "
                "(or __graft_entry__.build()); there is no CPU fallback")
        L = C.CDLL(path)
        vp, u64, sz, i = C.c_void_p, C.c_uint64, C.c_size_t, C.c_int
        cbp = C.POINTER(_CCodebook)
        L.splitzip_version.restype = i
        L.splitzip_strerror.restype = C.c_char_p
        L.splitzip_strerror.argtypes = [i]
        L.splitzip_calibrate.restype = i
        L.splitzip_calibrate.argtypes = [vp, u64, i, cbp, C.POINTER(C.c_uint64)]
        L.splitzip_codebook_from_dec.restype = i
        L.splitzip_codebook_from_dec.argtypes = [C.POINTER(C.c_uint8), i, cbp]
        for f in (L.splitzip_fixed_bytes, L.splitzip_compress_bound, L.splitzip_workspace_bytes):
            f.restype = sz
            f.argtypes = [u64, i]
        L.splitzip_total_bytes.restype = sz
        L.splitzip_total_bytes.argtypes = [u64, u64, i]
        L.splitzip_workspace_init.restype = i
        L.splitzip_workspace_init.argtypes = [vp, sz, vp]
        L.splitzip_compress.restype = i
        L.splitzip_compress.argtypes = [vp, u64, i, cbp, vp, sz, vp, sz, vp, vp]
        L.splitzip_decompress.restype = i
        L.splitzip_decompress.argtypes = [vp, sz, u64, i, cbp, vp, vp, vp]
        L.splitzip_codebook_from_hist.restype = i
        L.splitzip_codebook_from_hist.argtypes = [C.POINTER(C.c_uint64), i, cbp]
        L.splitzip_histogram.restype = i
        L.splitzip_histogram.argtypes = [vp, u64, i, vp, vp]
        L.splitzip_codebook_device.restype = i
        L.splitzip_codebook_device.argtypes = [vp, i, vp, vp]
        L.splitzip_compress_dcb.restype = i
        L.splitzip_compress_dcb.argtypes = [vp, u64, i, vp, vp, sz, vp, sz, vp, vp]
        L.splitzip_decompress_dcb.restype = i
        L.splitzip_decompress_dcb.argtypes = [vp, sz, u64, i, vp, vp, vp, vp]
        L.splitzip_compress_batch.restype = i
        L.splitzip_compress_batch.argtypes = [C.POINTER(_CItem), C.c_uint32, i, vp, sz, vp, vp]
        L.splitzip_decompress_batch.restype = i
        L.splitzip_decompress_batch.argtypes = [C.POINTER(_CDItem), C.c_uint32, i, vp, vp]
        L.splitzip_calibrate_batch_device.restype = i
        L.splitzip_calibrate_batch_device.argtypes = [C.POINTER(_CItem), C.c_uint32, i, vp, vp, vp]
        L.splitzip_compress_batch_dcb.restype = i
        L.splitzip_compress_batch_dcb.argtypes = [C.POINTER(_CItem), C.c_uint32, i, vp, vp, sz, vp, vp]
        L.splitzip_decompress_batch_dcb.restype = i
        L.splitzip_decompress_batch_dcb.argtypes = [C.POINTER(_CDItem), C.c_uint32, i, vp, vp, vp]
        L.splitzip_decompress_own.restype = i
        L.splitzip_decompress_own.argtypes = [vp, sz, u64, i, vp, vp, vp]
        L.splitzip_decompress_batch_own.restype = i
        L.splitzip_decompress_batch_own.argtypes = [C.POINTER(_CDItem), C.c_uint32, i, vp, vp]
        L.splitzip_noalloc_max_elems.restype = u64
        L.splitzip_noalloc_max_elems.argtypes = []
        L.splitzip_compress_noalloc.restype = i
        L.splitzip_compress_noalloc.argtypes = [vp, u64, i, cbp, vp, sz, vp, vp]
        L.splitzip_internal_test_hooks.restype = None
        L.splitzip_internal_test_hooks.argtypes = [u64, u64, C.c_uint32, u64]
        L.splitzip_internal_test_short.restype = None
        L.splitzip_internal_test_short.argtypes = [C.c_uint32, C.c_uint32]
        L.splitzip_internal_test_launch.restype = None
        L.splitzip_internal_test_launch.argtypes = [C.c_uint32, C.c_uint32, C.c_uint32]
        L.splitzip_internal_compress_plan.restype = None
        L.splitzip_internal_compress_plan.argtypes = [C.POINTER(_CItem), C.c_uint32, i, C.c_uint32, C.POINTER(C.c_uint32)]
        L.splitzip_internal_decompress_plan.restype = None
        L.splitzip_internal_decompress_plan.argtypes = [C.POINTER(_CDItem), C.c_uint32, i, C.POINTER(C.c_uint32)]
        L.splitzip_internal_stream_room.restype = C.c_uint32
        L.splitzip_internal_stream_room.argtypes = [u64, u64, i]
        L.splitzip_internal_calibrate_launches.restype = C.c_uint32
        L.splitzip_internal_calibrate_launches.argtypes = [C.POINTER(_CItem), C.c_uint32, i]
        L.splitzip_internal_calibrate_waits.restype = i
        L.splitzip_internal_calibrate_waits.argtypes = [u64, u64]
        L.splitzip_internal_xcd_tile.restype = C.c_uint32
        L.splitzip_internal_xcd_tile.argtypes = [C.c_uint32, C.c_uint32]
        L.splitzip_traffic_probe.restype = i
        L.splitzip_traffic_probe.argtypes = [vp, sz, vp, sz, vp]
        L.splitzip_traffic_probe_shape.restype = i
        L.splitzip_traffic_probe_shape.argtypes = [vp, sz, vp, sz, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32, vp]
        pgp = C.POINTER(_CPaged)
        L.splitzip_compress_paged.restype = i
        L.splitzip_compress_paged.argtypes = [pgp, u64, i, cbp, vp, sz, vp, sz, vp, vp]
        L.splitzip_decompress_paged.restype = i
        L.splitzip_decompress_paged.argtypes = [vp, sz, u64, i, cbp, pgp, vp, vp]
        L.splitzip_compress_batch_paged.restype = i
        L.splitzip_compress_batch_paged.argtypes = [C.POINTER(_CItem), C.c_uint32, i, pgp, vp, sz, vp, vp]
        L.splitzip_decompress_batch_paged.restype = i
        L.splitzip_decompress_batch_paged.argtypes = [C.POINTER(_CDItem), C.c_uint32, i, pgp, vp, vp]
        vrp = C.POINTER(Variant)
        L.splitzip_variant_supported.restype = i
        L.splitzip_variant_supported.argtypes = [vrp]
        L.splitzip_variant_total_bytes.restype = sz
        L.splitzip_variant_total_bytes.argtypes = [u64, u64, vrp]
        for f in (L.splitzip_variant_compress_bound, L.splitzip_variant_workspace_bytes):
            f.restype = sz
            f.argtypes = [u64, vrp]
        L.splitzip_variant_calibrate.restype = i
        L.splitzip_variant_calibrate.argtypes = [vp, u64, vrp, cbp, C.POINTER(C.c_uint64)]
        L.splitzip_variant_codebook_from_dec.restype = i
        L.splitzip_variant_codebook_from_dec.argtypes = [C.POINTER(C.c_uint8), vrp, cbp]
        L.splitzip_variant_compress.restype = i
        L.splitzip_variant_compress.argtypes = [vp, u64, vrp, cbp, vp, sz, vp, sz, vp, vp]
        L.splitzip_variant_decompress.restype = i
        L.splitzip_variant_decompress.argtypes = [vp, sz, u64, vrp, cbp, vp, vp, vp]
        chp, sqp = C.POINTER(_CCache), C.POINTER(_CSeqs)
        for f in (L.splitzip_cache_write, L.splitzip_cache_read):
            f.restype = i
            f.argtypes = [chp, sqp, vp, u64, vp, u64, C.c_uint32, vp]
        L.splitzip_attention_workspace_bytes.restype = sz
        L.splitzip_attention_workspace_bytes.argtypes = [chp, sqp, C.c_uint32, C.c_uint32]
        L.splitzip_cache_attention.restype = i
        L.splitzip_cache_attention.argtypes = [chp, sqp, C.POINTER(_CAttention), vp, u64, vp, u64, vp, C.c_uint32, C.c_uint32, vp, sz, vp]
        L.splitzip_cache_append.restype = i
        L.splitzip_cache_append.argtypes = [chp, sqp, C.POINTER(_CRotation), *[vp, u64] * 5, C.c_uint32, C.c_uint32, vp]
        L.splitzip_cache_allot.restype = i
        L.splitzip_cache_allot.argtypes = [C.POINTER(_CPool), sqp, vp, vp, vp, vp, vp, C.c_uint32, vp]
        L.splitzip_cache_move.restype = i
        L.splitzip_cache_move.argtypes = [chp, C.c_uint32, sqp, vp, C.c_uint32, C.c_uint32, vp]
        L.fast, L.fast_cache = _short_way(L)
        _lib = L
        _leave_fast_in_a_bad_fork()
    return _lib


def _short_way(L):
    """The functions of _fastcall, the codec's and the cache's, or, where it is not built or built for another Python or torch, none that
    take a call."""
    try:
        from . import _fastcall   # torch's own libraries are loaded by now
        of = _fastcall.bind(L._handle, _CCodebook, Variant, _CPaged, _CCache, _CSeqs, _CAttentionOf, _CRotationOf, _CPool, torch.__version__)
        cache = {name: of.pop(name) for name in list(of) if name.startswith("splitzip_cache_")}
        return types.SimpleNamespace(**of), types.SimpleNamespace(**cache)
    except ImportError as e:
        warnings.warn(f"{e}: calls take the general way, 1 to 2 us longer each; build the short one with "
                      "`python -m paper_2605_01708_amd.build`", RuntimeWarning, stacklevel=3)
        return _NoneTaken(), _NoneTaken()


class _NoneTaken:
    """lib().fast, or fast_cache, where every call goes the general way."""

    def __getattr__(self, name):
        return lambda *args: _NOT_TAKEN


def _leave_fast_in_a_bad_fork() -> None:
    """In a child of a process that had used the GPU before it forked, torch refuses the GPU where the general way asks it for
    the current stream; the short way does not ask torch."""
    if _lib is not None and getattr(torch._C, "_cuda_isInBadFork", bool)():
        _lib.fast = _lib.fast_cache = _NoneTaken()


if hasattr(os, "register_at_fork"):
    os.register_at_fork(after_in_child=_leave_fast_in_a_bad_fork)


def _check(rc: int, what: str):
    if rc != 0:
        raise SplitZipError(rc, what)


_NOT_TAKEN = 1   # what a function of lib().fast answers if it has done nothing


def _handle(stream):
    """What lib().fast takes for a stream, its handle; for the current one it takes None.  (The calls below have neither a
    call of their own for that, nor one for a result of 0 or for the library that is loaded: 0.1 us each.)"""
    return int(stream.cuda_stream)


class Codebook:
    """Host-side calibration tables (a splitzip_codebook)."""

    def __init__(self, c: _CCodebook):
        self.c = c

    @property
    def dtype(self) -> int:
        return int(self.c.dtype)

    @property
    def dec(self):
        return list(self.c.dec)

    @property
    def enc(self):
        return list(self.c.enc)

    @property
    def member(self):
        return list(self.c.member)


def _elem_size(dtype: int) -> int:
    return 2 if dtype == BF16 else 1


def calibrate(sample: torch.Tensor, dtype: int, return_hist: bool = False):
    """splitzip_calibrate on a HOST tensor of raw words (any 2-byte dtype for BF16, 1-byte for E5M2)."""
    if sample.device.type != "cpu":
        raise ValueError("calibration runs on the host: pass a CPU tensor")
    s = sample.contiguous()
    if s.element_size() != _elem_size(dtype):
        raise ValueError("sample element size does not match dtype")
    cb = _CCodebook()
    hist = (C.c_uint64 * 256)()
    _check(lib().splitzip_calibrate(s.data_ptr(), s.numel(), dtype, C.byref(cb), hist), "splitzip_calibrate")
    return (Codebook(cb), list(hist)) if return_hist else Codebook(cb)


def codebook_from_dec(dec, dtype: int) -> Codebook:
    arr = (C.c_uint8 * 16)(*[int(v) for v in dec])
    cb = _CCodebook()
    _check(lib().splitzip_codebook_from_dec(arr, dtype, C.byref(cb)), "splitzip_codebook_from_dec")
    return Codebook(cb)


def codebook_from_hist(hist, dtype: int) -> Codebook:
    """splitzip_codebook_from_hist on a host list / tensor of 256 exponent counts."""
    vals = [int(v) for v in (hist.tolist() if hasattr(hist, "tolist") else hist)]
    arr = (C.c_uint64 * 256)(*vals)
    cb = _CCodebook()
    _check(lib().splitzip_codebook_from_hist(arr, dtype, C.byref(cb)), "splitzip_codebook_from_hist")
    return Codebook(cb)


def histogram(x: torch.Tensor, dtype: int, hist: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """splitzip_histogram: adds the exponent counts of the device words x to hist (256 x int64 on the
    device; a zeroed one is made if none is given) and returns it."""
    if x.element_size() != _elem_size(dtype) or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of raw words of the dtype")
    if hist is None:
        hist = torch.zeros(256, dtype=torch.int64, device=x.device)
    _check(lib().splitzip_histogram(x.data_ptr(), x.numel(), dtype, hist.data_ptr(), _stream_ptr(stream)), "splitzip_histogram")
    return hist


class DeviceCodebook:
    """A splitzip_codebook in device memory, written by splitzip_codebook_device."""

    def __init__(self, dtype: int, device="cuda"):
        self.dtype = dtype
        self.buf = torch.zeros((C.sizeof(_CCodebook) + 7) // 8, dtype=torch.int64, device=device)

    def to_host(self) -> Codebook:
        """Copy of the tables on the host (synchronises)."""
        raw = self.buf.cpu().numpy().tobytes()[: C.sizeof(_CCodebook)]
        return Codebook(_CCodebook.from_buffer_copy(raw))


def codebook_device(hist: torch.Tensor, dtype: int, out: DeviceCodebook | None = None, stream=None) -> DeviceCodebook:
    """splitzip_codebook_device: the tables for 256 device counts, written to device memory."""
    out = DeviceCodebook(dtype, hist.device) if out is None else out
    _check(lib().splitzip_codebook_device(hist.data_ptr(), dtype, out.buf.data_ptr(), _stream_ptr(stream)), "splitzip_codebook_device")
    return out


def compress_dcb(x: torch.Tensor, d_cb: DeviceCodebook, out: torch.Tensor, workspace: "Workspace", sizes: torch.Tensor,
                 stream=None, capacity: int | None = None) -> None:
    """splitzip_compress_dcb: splitzip_compress with a codebook in device memory."""
    rc = (_lib or lib()).fast.splitzip_compress_dcb(x, d_cb.dtype, d_cb.buf, out, capacity, workspace.buf, workspace.nbytes, sizes,
                                          None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_compress_dcb") if rc else None
    if x.element_size() != _elem_size(d_cb.dtype) or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of raw words of the codebook's dtype")
    cap = out.numel() * out.element_size() if capacity is None else capacity
    _check(lib().splitzip_compress_dcb(x.data_ptr(), x.numel(), d_cb.dtype, d_cb.buf.data_ptr(), out.data_ptr(), cap,
                                       workspace.buf.data_ptr(), workspace.nbytes, sizes.data_ptr(), _stream_ptr(stream)),
           "splitzip_compress_dcb")


def decompress_dcb(comp: torch.Tensor, comp_bytes: int, n_elems: int, d_cb: DeviceCodebook, out: torch.Tensor,
                   sizes: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_decompress_dcb: splitzip_decompress with a codebook in device memory."""
    rc = (_lib or lib()).fast.splitzip_decompress_dcb(comp, comp_bytes, n_elems, d_cb.dtype, d_cb.buf, out, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_decompress_dcb") if rc else None
    if out.numel() < n_elems or out.element_size() != _elem_size(d_cb.dtype) or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of at least n_elems raw words")
    _check(lib().splitzip_decompress_dcb(comp.data_ptr(), comp_bytes, n_elems, d_cb.dtype, d_cb.buf.data_ptr(), out.data_ptr(),
                                         sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
           "splitzip_decompress_dcb")


def fixed_bytes(n: int, dtype: int) -> int:
    return int(lib().splitzip_fixed_bytes(n, dtype))


def total_bytes(n: int, m: int, dtype: int) -> int:
    return int(lib().splitzip_total_bytes(n, m, dtype))


def compress_bound(n: int, dtype: int) -> int:
    return int(lib().splitzip_compress_bound(n, dtype))


def workspace_bytes(n: int, dtype: int) -> int:
    return int(lib().splitzip_workspace_bytes(n, dtype))


# The handle of the current stream without a torch.cuda.Stream object around it: making one costs 2.7 us a call, as
# much as a kernel launch; the handle alone 0.3 us.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    if _raw_stream is not None:
        return int(_raw_stream(torch.cuda.current_device()))
    return int(torch.cuda.current_stream().cuda_stream)


class Workspace:
    """Device scratch for compress calls of up to n_elems; initialised once."""

    def __init__(self, n_elems: int, dtype: int, device="cuda", stream=None):
        self.n_elems = n_elems
        self.nbytes = workspace_bytes(n_elems, dtype)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        _check(lib().splitzip_workspace_init(self.buf.data_ptr(), self.nbytes, _stream_ptr(stream)),
               "splitzip_workspace_init")


def new_sizes(device="cuda") -> torch.Tensor:
    """Zeroed device splitzip_sizes record (24 bytes as 3 x int64)."""
    return torch.zeros(3, dtype=torch.int64, device=device)


def read_sizes(sizes: torch.Tensor):
    """(total_bytes, n_escapes, status) -- copies the record to the host (synchronises)."""
    h = sizes.cpu()
    return int(h[0]), int(h[1]), int(h[2]) & 0xFFFFFFFF


def compress(x: torch.Tensor, cb: Codebook, out: torch.Tensor, workspace: Workspace,
             sizes: torch.Tensor, stream=None, capacity: int | None = None) -> None:
    """splitzip_compress: x (device words) -> out (device uint8), sizes written on the stream."""
    rc = (_lib or lib()).fast.splitzip_compress(x, cb.c, out, capacity, workspace.buf, workspace.nbytes, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_compress") if rc else None
    n = x.numel()
    if x.element_size() != _elem_size(cb.dtype) or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of raw words of the codebook's dtype")
    cap = out.numel() * out.element_size() if capacity is None else capacity
    _check(lib().splitzip_compress(x.data_ptr(), n, cb.dtype, C.byref(cb.c), out.data_ptr(), cap,
                                   workspace.buf.data_ptr(), workspace.nbytes, sizes.data_ptr(),
                                   _stream_ptr(stream)), "splitzip_compress")


def internal_test_hooks(stage_bytes: int = 0, status_bytes: int = 0, finish_groups: int = 0, direct_bytes: int = 0) -> None:
    """What the tests of the rarely taken paths turn (not part of splitzip.h): a staging area and a status area smaller
    than the workspace has, the groups of tiles per workgroup of the finishing pass (1, 2 or 4), and the bytes of tile
    counts a launch's finishing pass may read directly (beyond: sums of 64 counts).  0 = as built."""
    lib().splitzip_internal_test_hooks(stage_bytes, status_bytes, finish_groups, direct_bytes)


def internal_test_launch(cpt: int = 0, cpw: int = 0, xcd: int = 0) -> None:
    """Forces what the launch rules choose by size (not part of splitzip.h): chunks per wave of the compress tiles (cpt) and
    of the decoders (cpw), 1, 2, 4 or 8, and the tiles' order in batch launches (xcd: 1 their own, 2 xcd_order).
    0 = by the rules."""
    lib().splitzip_internal_test_launch(cpt, cpw, xcd)


def internal_test_short(looks: int = 0, anywhere: bool = False) -> None:
    """How often a workgroup of a short compress launch looks for the others' counts before it leaves its tile to them, and whether
    there are such launches on streams whose share of the device does not hold them (not part of splitzip.h).  0 = as built;
    INTERNAL_NO_SHORT: two launches instead."""
    lib().splitzip_internal_test_short(looks, anywhere)


INTERNAL_NO_SHORT = 0xFFFFFFFF


def internal_compress_plan(n_elems, dtype: int, cus: int = 256) -> dict:
    """How a compress call's first launch over tensors of these lengths is shaped under capture, and, otherwise, the chunks per wave
    of compress_short_kernel if that takes them on a stream of so many CUs (host only, for tests of the rules)."""
    items, out = (_CItem * len(n_elems))(), (C.c_uint32 * 9)()
    for it, n in zip(items, n_elems):
        it.n_elems = n
    lib().splitzip_internal_compress_plan(items, len(n_elems), dtype, cus, out)
    return dict(zip(("tensors", "cpt", "tiles_max", "launches", "by_xcd", "finish_groups", "group_sums", "small", "short"), out))


def internal_decompress_plan(n_elems, dtype: int, comp_bytes=None) -> dict:
    """The same for a batch decompress call (comp_bytes: of the streams; by default those of streams without escapes)."""
    items, out = (_CDItem * len(n_elems))(), (C.c_uint32 * 4)()
    for k, (it, n) in enumerate(zip(items, n_elems)):
        it.n_elems, it.comp_bytes = n, fixed_bytes(n, dtype) if comp_bytes is None else comp_bytes[k]
    lib().splitzip_internal_decompress_plan(items, len(n_elems), dtype, out)
    return dict(zip(("cpw", "workgroups", "by_xcd", "lds_pad"), out))


def internal_stream_room(comp_bytes: int, n_elems: int, dtype: int) -> int:
    """The escapes that a stream of comp_bytes bytes (its fixed part at least) has room for, n_elems at most (for tests)."""
    return int(lib().splitzip_internal_stream_room(comp_bytes, n_elems, dtype))


def internal_xcd_tile(workgroup: int, n_tiles: int) -> int:
    """The tile that a workgroup of a tensor of n_tiles tiles takes in a launch that goes by XCDs (for tests)."""
    return int(lib().splitzip_internal_xcd_tile(workgroup, n_tiles))


def internal_calibrate_launches(n_elems, dtype: int) -> int:
    """The launches of a calibration call over samples of these lengths (host only, for tests of the rules)."""
    items = (_CItem * len(n_elems))()
    for it, n in zip(items, n_elems):
        it.n_elems = n
    return int(lib().splitzip_internal_calibrate_launches(items, len(n_elems), dtype))


def internal_calibrate_waits(word: int, tag: int) -> bool:
    """Whether a workgroup of the calibration call `tag` waits where it finds `word` (for tests)."""
    return bool(lib().splitzip_internal_calibrate_waits(word, tag))


def noalloc_max_elems() -> int:
    return int(lib().splitzip_noalloc_max_elems())


def compress_noalloc(x: torch.Tensor, cb: Codebook, out: torch.Tensor, sizes: torch.Tensor, stream=None,
                     capacity: int | None = None) -> None:
    """splitzip_compress_noalloc: splitzip_compress on the library's own per-GPU scratch array instead of a workspace."""
    rc = (_lib or lib()).fast.splitzip_compress_noalloc(x, cb.c, out, capacity, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_compress_noalloc") if rc else None
    n = x.numel()
    if x.element_size() != _elem_size(cb.dtype) or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of raw words of the codebook's dtype")
    cap = out.numel() * out.element_size() if capacity is None else capacity
    _check(lib().splitzip_compress_noalloc(x.data_ptr(), n, cb.dtype, C.byref(cb.c), out.data_ptr(), cap,
                                           sizes.data_ptr(), _stream_ptr(stream)), "splitzip_compress_noalloc")


def decompress(comp: torch.Tensor, comp_bytes: int, n_elems: int, cb: Codebook, out: torch.Tensor,
               sizes: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_decompress: comp (device uint8 stream) -> out (device words)."""
    rc = (_lib or lib()).fast.splitzip_decompress(comp, comp_bytes, n_elems, cb.c, out, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_decompress") if rc else None
    if out.numel() < n_elems or out.element_size() != _elem_size(cb.dtype) or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of at least n_elems raw words")
    _check(lib().splitzip_decompress(comp.data_ptr(), comp_bytes, n_elems, cb.dtype, C.byref(cb.c),
                                     out.data_ptr(), sizes.data_ptr() if sizes is not None else None,
                                     _stream_ptr(stream)), "splitzip_decompress")


def new_sizes_array(n: int, device="cuda") -> torch.Tensor:
    """n zeroed device splitzip_sizes records, one row of 3 x int64 each."""
    return torch.zeros(n, 3, dtype=torch.int64, device=device)


def read_sizes_array(sizes: torch.Tensor):
    """[(total_bytes, n_escapes, status), ...] -- copies to the host (synchronises)."""
    h = sizes.cpu().tolist()
    return [(int(r[0]), int(r[1]), int(r[2]) & 0xFFFFFFFF) for r in h]


class CompressBatch:
    """The marshalled item list of a splitzip_compress_batch call; build once, launch many times."""

    def __init__(self, xs, cbs, outs, capacities=None):
        if not (len(xs) == len(cbs) == len(outs)):
            raise ValueError("xs, cbs and outs must have the same length")
        self.n = len(xs)
        self.dtype = cbs[0].dtype if cbs else BF16
        self.items = (_CItem * max(self.n, 1))()
        self._keep = (list(xs), list(cbs), list(outs))
        for k, (x, cb, out) in enumerate(zip(xs, cbs, outs)):
            if x.element_size() != _elem_size(cb.dtype) or not x.is_contiguous() or cb.dtype != self.dtype:
                raise ValueError("every x must be a contiguous tensor of raw words of one dtype")
            cap = out.numel() * out.element_size() if capacities is None else capacities[k]
            self.items[k] = _CItem(x.data_ptr(), x.numel(), out.data_ptr(), cap, C.pointer(cb.c))

    def launch(self, workspace: "Workspace", sizes: torch.Tensor, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_compress_batch(self.items, self.n, self.dtype, workspace.buf, workspace.nbytes, sizes,
                                                None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_compress_batch") if rc else None
        _check(lib().splitzip_compress_batch(self.items, self.n, self.dtype, workspace.buf.data_ptr(), workspace.nbytes,
                                             sizes.data_ptr(), _stream_ptr(stream)), "splitzip_compress_batch")


class DecompressBatch:
    """The marshalled item list of a splitzip_decompress_batch call."""

    def __init__(self, comps, comp_bytes, n_elems, cbs, outs):
        if not (len(comps) == len(comp_bytes) == len(n_elems) == len(cbs) == len(outs)):
            raise ValueError("all lists must have the same length")
        self.n = len(comps)
        self.dtype = cbs[0].dtype if cbs else BF16
        self.items = (_CDItem * max(self.n, 1))()
        self._keep = (list(comps), list(cbs), list(outs))
        for k, (c, cbytes, n, cb, out) in enumerate(zip(comps, comp_bytes, n_elems, cbs, outs)):
            if out.numel() < n or out.element_size() != _elem_size(cb.dtype) or not out.is_contiguous() or cb.dtype != self.dtype:
                raise ValueError("every out must be a contiguous tensor of at least n_elems raw words of one dtype")
            self.items[k] = _CDItem(c.data_ptr(), cbytes, n, out.data_ptr(), C.pointer(cb.c))

    def launch(self, sizes: torch.Tensor | None = None, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_decompress_batch(self.items, self.n, self.dtype, sizes, None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_decompress_batch") if rc else None
        _check(lib().splitzip_decompress_batch(self.items, self.n, self.dtype,
                                               sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
               "splitzip_decompress_batch")


class DeviceCodebooks:
    """n splitzip_codebook in device memory, written by splitzip_calibrate_batch_device, and the counts they come from."""

    def __init__(self, n: int, dtype: int, device="cuda"):
        self.n, self.dtype = n, dtype
        self.buf = torch.zeros(max(n, 1) * C.sizeof(_CCodebook) // 4, dtype=torch.int32, device=device)
        self.hists = torch.zeros((max(n, 1), 256), dtype=torch.int64, device=device)

    def to_host(self, k: int) -> Codebook:
        """Copy of the k-th codebook on the host (synchronises)."""
        w = C.sizeof(_CCodebook) // 4
        raw = self.buf[k * w:(k + 1) * w].cpu().numpy().tobytes()
        return Codebook(_CCodebook.from_buffer_copy(raw))


def _null_cb():
    return C.POINTER(_CCodebook)()


class CalibrateBatchDevice:
    """splitzip_calibrate_batch_device: a codebook per tensor, counted and ranked on the device."""

    def __init__(self, xs, dcbs: DeviceCodebooks):
        self.n, self.dcbs = len(xs), dcbs
        self.items = (_CItem * max(self.n, 1))()
        self._keep = list(xs)
        for k, x in enumerate(xs):
            if x.element_size() != _elem_size(dcbs.dtype) or not x.is_contiguous():
                raise ValueError("every x must be a contiguous tensor of raw words of the codebooks' dtype")
            self.items[k] = _CItem(x.data_ptr(), x.numel(), None, 0, _null_cb())

    def launch(self, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_calibrate_batch_device(self.items, self.n, self.dcbs.dtype, self.dcbs.hists,
                                                        self.dcbs.buf, None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_calibrate_batch_device") if rc else None
        _check(lib().splitzip_calibrate_batch_device(self.items, self.n, self.dcbs.dtype, self.dcbs.hists.data_ptr(),
                                                     self.dcbs.buf.data_ptr(), _stream_ptr(stream)), "splitzip_calibrate_batch_device")


class CompressBatchDcb:
    """splitzip_compress_batch_dcb: tensor k under the k-th codebook of a DeviceCodebooks."""

    def __init__(self, xs, dcbs: DeviceCodebooks, outs, capacities=None):
        if not (len(xs) == len(outs)) or len(xs) > dcbs.n:
            raise ValueError("xs and outs must have the same length, at most the number of codebooks")
        self.n, self.dcbs = len(xs), dcbs
        self.items = (_CItem * max(self.n, 1))()
        self._keep = (list(xs), list(outs))
        for k, (x, out) in enumerate(zip(xs, outs)):
            if x.element_size() != _elem_size(dcbs.dtype) or not x.is_contiguous():
                raise ValueError("every x must be a contiguous tensor of raw words of the codebooks' dtype")
            cap = out.numel() * out.element_size() if capacities is None else capacities[k]
            self.items[k] = _CItem(x.data_ptr(), x.numel(), out.data_ptr(), cap, _null_cb())

    def launch(self, workspace: "Workspace", sizes: torch.Tensor, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_compress_batch_dcb(self.items, self.n, self.dcbs.dtype, self.dcbs.buf, workspace.buf,
                                                    workspace.nbytes, sizes, None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_compress_batch_dcb") if rc else None
        _check(lib().splitzip_compress_batch_dcb(self.items, self.n, self.dcbs.dtype, self.dcbs.buf.data_ptr(),
                                                 workspace.buf.data_ptr(), workspace.nbytes, sizes.data_ptr(),
                                                 _stream_ptr(stream)), "splitzip_compress_batch_dcb")


class DecompressBatchDcb:
    """splitzip_decompress_batch_dcb: stream k under the k-th codebook of a DeviceCodebooks."""

    def __init__(self, comps, comp_bytes, n_elems, dcbs: DeviceCodebooks, outs):
        if not (len(comps) == len(comp_bytes) == len(n_elems) == len(outs)) or len(comps) > dcbs.n:
            raise ValueError("all lists must have the same length, at most the number of codebooks")
        self.n, self.dcbs = len(comps), dcbs
        self.items = (_CDItem * max(self.n, 1))()
        self._keep = (list(comps), list(outs))
        for k, (c, cbytes, n, out) in enumerate(zip(comps, comp_bytes, n_elems, outs)):
            if out.numel() < n or out.element_size() != _elem_size(dcbs.dtype) or not out.is_contiguous():
                raise ValueError("every out must be a contiguous tensor of at least n_elems raw words of the codebooks' dtype")
            self.items[k] = _CDItem(c.data_ptr(), cbytes, n, out.data_ptr(), _null_cb())

    def launch(self, sizes: torch.Tensor | None = None, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_decompress_batch_dcb(self.items, self.n, self.dcbs.dtype, self.dcbs.buf, sizes,
                                                      None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_decompress_batch_dcb") if rc else None
        _check(lib().splitzip_decompress_batch_dcb(self.items, self.n, self.dcbs.dtype, self.dcbs.buf.data_ptr(),
                                                   sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
               "splitzip_decompress_batch_dcb")


def decompress_own(comp: torch.Tensor, comp_bytes: int, n_elems: int, dtype: int, out: torch.Tensor,
                   sizes: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_decompress_own: decompress with the codebook the stream carries in its header."""
    rc = (_lib or lib()).fast.splitzip_decompress_own(comp, comp_bytes, n_elems, dtype, out, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_decompress_own") if rc else None
    if out.numel() < n_elems or out.element_size() != _elem_size(dtype) or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of at least n_elems raw words of the dtype")
    _check(lib().splitzip_decompress_own(comp.data_ptr(), comp_bytes, n_elems, dtype, out.data_ptr(),
                                         sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
           "splitzip_decompress_own")


class DecompressBatchOwn:
    """splitzip_decompress_batch_own: every stream under the codebook of its own header."""

    def __init__(self, comps, comp_bytes, n_elems, dtype: int, outs):
        if not (len(comps) == len(comp_bytes) == len(n_elems) == len(outs)):
            raise ValueError("all lists must have the same length")
        self.n, self.dtype = len(comps), dtype
        self.items = (_CDItem * max(self.n, 1))()
        self._keep = (list(comps), list(outs))
        for k, (c, cbytes, n, out) in enumerate(zip(comps, comp_bytes, n_elems, outs)):
            if out.numel() < n or out.element_size() != _elem_size(dtype) or not out.is_contiguous():
                raise ValueError("every out must be a contiguous tensor of at least n_elems raw words of the dtype")
            self.items[k] = _CDItem(c.data_ptr(), cbytes, n, out.data_ptr(), _null_cb())

    def launch(self, sizes: torch.Tensor | None = None, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_decompress_batch_own(self.items, self.n, self.dtype, sizes, None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_decompress_batch_own") if rc else None
        _check(lib().splitzip_decompress_batch_own(self.items, self.n, self.dtype,
                                                   sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
               "splitzip_decompress_batch_own")


def compress_batch(xs, cbs, outs, workspace: Workspace, sizes: torch.Tensor, stream=None, capacities=None) -> None:
    """splitzip_compress_batch: xs[k] -> outs[k] with codebook cbs[k]; sizes = new_sizes_array(len(xs))."""
    CompressBatch(xs, cbs, outs, capacities).launch(workspace, sizes, stream)


def decompress_batch(comps, comp_bytes, n_elems, cbs, outs, sizes: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_decompress_batch: comps[k] (comp_bytes[k] bytes, n_elems[k] words) -> outs[k]."""
    DecompressBatch(comps, comp_bytes, n_elems, cbs, outs).launch(sizes, stream)


def traffic_probe(src: torch.Tensor, read_bytes: int, dst: torch.Tensor, write_bytes: int, stream=None) -> None:
    _check(lib().splitzip_traffic_probe(src.data_ptr(), read_bytes, dst.data_ptr(), write_bytes,
                                        _stream_ptr(stream)), "splitzip_traffic_probe")


def traffic_probe_shape(src: torch.Tensor, read_bytes: int, dst: torch.Tensor, write_bytes: int, reads_per_step: int,
                        writes_per_step: int, wgs_per_cu: int, flags: int = 3, stream=None) -> None:
    _check(lib().splitzip_traffic_probe_shape(src.data_ptr(), read_bytes, dst.data_ptr(), write_bytes, reads_per_step,
                                              writes_per_step, wgs_per_cu, flags, _stream_ptr(stream)),
           "splitzip_traffic_probe_shape")


# ---- format variants of the ablations -----------------------------------------------------------

def variant(dtype: int, code_bits: int = 4, k: int = 16, escape_mode: int = 0, chunk_elems: int = 1024,
            value_bits: int = 0) -> Variant:
    return Variant(dtype, code_bits, k, escape_mode, chunk_elems, value_bits)


def variant_supported(v: Variant) -> bool:
    return bool(lib().splitzip_variant_supported(C.byref(v)))


def variant_total_bytes(n: int, m: int, v: Variant) -> int:
    return int(lib().splitzip_variant_total_bytes(n, m, C.byref(v)))


def variant_compress_bound(n: int, v: Variant) -> int:
    return int(lib().splitzip_variant_compress_bound(n, C.byref(v)))


def variant_workspace_bytes(n: int, v: Variant) -> int:
    return int(lib().splitzip_variant_workspace_bytes(n, C.byref(v)))


def variant_calibrate(sample: torch.Tensor, v: Variant, return_hist: bool = False):
    """splitzip_variant_calibrate on a HOST tensor of raw words."""
    if sample.device.type != "cpu":
        raise ValueError("calibration runs on the host: pass a CPU tensor")
    s = sample.contiguous()
    if s.element_size() != _elem_size(v.dtype):
        raise ValueError("sample element size does not match dtype")
    cb = _CCodebook()
    hist = (C.c_uint64 * 256)()
    _check(lib().splitzip_variant_calibrate(s.data_ptr(), s.numel(), C.byref(v), C.byref(cb), hist),
           "splitzip_variant_calibrate")
    return (Codebook(cb), list(hist)) if return_hist else Codebook(cb)


def variant_codebook_from_dec(dec, v: Variant) -> Codebook:
    vals = [int(x) for x in dec][:16]
    arr = (C.c_uint8 * 16)(*(vals + [0] * (16 - len(vals))))
    cb = _CCodebook()
    _check(lib().splitzip_variant_codebook_from_dec(arr, C.byref(v), C.byref(cb)), "splitzip_variant_codebook_from_dec")
    return Codebook(cb)


def variant_compress(x: torch.Tensor, v: Variant, cb: Codebook, out: torch.Tensor, workspace: torch.Tensor,
                     sizes: torch.Tensor, stream=None, capacity: int | None = None) -> None:
    """splitzip_variant_compress; workspace is a device uint8 tensor of variant_workspace_bytes."""
    rc = (_lib or lib()).fast.splitzip_variant_compress(x, v, cb.c, out, capacity, workspace, None, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_variant_compress") if rc else None
    if x.element_size() != _elem_size(v.dtype) or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of raw words of the variant's dtype")
    cap = out.numel() * out.element_size() if capacity is None else capacity
    _check(lib().splitzip_variant_compress(x.data_ptr(), x.numel(), C.byref(v), C.byref(cb.c), out.data_ptr(), cap,
                                           workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                           sizes.data_ptr(), _stream_ptr(stream)), "splitzip_variant_compress")


def variant_decompress(comp: torch.Tensor, comp_bytes: int, n_elems: int, v: Variant, cb: Codebook, out: torch.Tensor,
                       sizes: torch.Tensor | None = None, stream=None) -> None:
    rc = (_lib or lib()).fast.splitzip_variant_decompress(comp, comp_bytes, n_elems, v, cb.c, out, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_variant_decompress") if rc else None
    if out.numel() < n_elems or out.element_size() != _elem_size(v.dtype) or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of at least n_elems raw words")
    _check(lib().splitzip_variant_decompress(comp.data_ptr(), comp_bytes, n_elems, C.byref(v), C.byref(cb.c),
                                             out.data_ptr(), sizes.data_ptr() if sizes is not None else None,
                                             _stream_ptr(stream)), "splitzip_variant_decompress")


# ---- paged / strided tensors ------------------------------------------------------------------------

class Paged:
    """splitzip_paged: a tensor whose words sit in pages of a pool, found through a block table.

    pool: device tensor (any dtype) holding the pages; block_table: device int32/uint32 tensor of page indices;
    block_elems: elements of this tensor per page; page_stride_bytes / offset_bytes as in include/splitzip.h."""

    def __init__(self, pool: torch.Tensor, block_table: torch.Tensor, block_elems: int, page_stride_bytes: int,
                 offset_bytes: int = 0, n_pool_blocks: int | None = None):
        if block_table.element_size() != 4 or not block_table.is_contiguous():
            raise ValueError("block_table must be a contiguous tensor of 32-bit page indices")
        self.pool, self.block_table = pool, block_table            # keep the tensors alive
        pool_bytes = pool.numel() * pool.element_size()
        npool = pool_bytes // page_stride_bytes if n_pool_blocks is None else n_pool_blocks
        self.c = _CPaged(pool.data_ptr(), block_table.data_ptr(), block_table.numel(), npool, block_elems, 0,
                         page_stride_bytes, offset_bytes)


def compress_paged(src: Paged, n_elems: int, cb: Codebook, out: torch.Tensor, workspace: Workspace,
                   sizes: torch.Tensor, stream=None, capacity: int | None = None) -> None:
    rc = (_lib or lib()).fast.splitzip_compress_paged(src.c, n_elems, cb.c, out, capacity, workspace.buf, workspace.nbytes, sizes,
                                            None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_compress_paged") if rc else None
    cap = out.numel() * out.element_size() if capacity is None else capacity
    _check(lib().splitzip_compress_paged(C.byref(src.c), n_elems, cb.dtype, C.byref(cb.c), out.data_ptr(), cap,
                                         workspace.buf.data_ptr(), workspace.nbytes, sizes.data_ptr(),
                                         _stream_ptr(stream)), "splitzip_compress_paged")


def decompress_paged(comp: torch.Tensor, comp_bytes: int, n_elems: int, cb: Codebook, dst: Paged,
                     sizes: torch.Tensor | None = None, stream=None) -> None:
    rc = (_lib or lib()).fast.splitzip_decompress_paged(comp, comp_bytes, n_elems, cb.c, dst.c, sizes, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_decompress_paged") if rc else None
    _check(lib().splitzip_decompress_paged(comp.data_ptr(), comp_bytes, n_elems, cb.dtype, C.byref(cb.c),
                                           C.byref(dst.c), sizes.data_ptr() if sizes is not None else None,
                                           _stream_ptr(stream)), "splitzip_decompress_paged")


class CompressBatchPaged:
    """splitzip_compress_batch_paged: tensors k = 0.. in pools that share one block table.  pools[k] is a device tensor
    whose first byte is the tensor's first word in page 0 (a view into the pool at the tensor's offset); n_elems[k] its
    logical length; paging a Paged that carries the table and the page geometry."""

    def __init__(self, pools, n_elems, cbs, outs, paging: Paged, capacities=None):
        if not (len(pools) == len(n_elems) == len(cbs) == len(outs)):
            raise ValueError("all lists must have the same length")
        self.n = len(pools)
        self.dtype = cbs[0].dtype if cbs else BF16
        self.paging = paging
        self.items = (_CItem * max(self.n, 1))()
        self._keep = (list(pools), list(cbs), list(outs))
        for k, (pool, n, cb, out) in enumerate(zip(pools, n_elems, cbs, outs)):
            cap = out.numel() * out.element_size() if capacities is None else capacities[k]
            self.items[k] = _CItem(pool.data_ptr(), n, out.data_ptr(), cap, C.pointer(cb.c))

    def launch(self, workspace: "Workspace", sizes: torch.Tensor, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_compress_batch_paged(self.items, self.n, self.dtype, self.paging.c, workspace.buf,
                                                      workspace.nbytes, sizes, None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_compress_batch_paged") if rc else None
        _check(lib().splitzip_compress_batch_paged(self.items, self.n, self.dtype, C.byref(self.paging.c),
                                                   workspace.buf.data_ptr(), workspace.nbytes, sizes.data_ptr(),
                                                   _stream_ptr(stream)), "splitzip_compress_batch_paged")


class DecompressBatchPaged:
    """splitzip_decompress_batch_paged: the reverse, into pools that share one block table."""

    def __init__(self, comps, comp_bytes, n_elems, cbs, pools, paging: Paged):
        if not (len(comps) == len(comp_bytes) == len(n_elems) == len(cbs) == len(pools)):
            raise ValueError("all lists must have the same length")
        self.n = len(comps)
        self.dtype = cbs[0].dtype if cbs else BF16
        self.paging = paging
        self.items = (_CDItem * max(self.n, 1))()
        self._keep = (list(comps), list(cbs), list(pools))
        for k, (c, cbytes, n, cb, pool) in enumerate(zip(comps, comp_bytes, n_elems, cbs, pools)):
            self.items[k] = _CDItem(c.data_ptr(), cbytes, n, pool.data_ptr(), C.pointer(cb.c))

    def launch(self, sizes: torch.Tensor | None = None, stream=None) -> None:
        rc = (_lib or lib()).fast.splitzip_decompress_batch_paged(self.items, self.n, self.dtype, self.paging.c, sizes,
                                                        None if stream is None else _handle(stream))
        if rc != _NOT_TAKEN:
            return _check(rc, "splitzip_decompress_batch_paged") if rc else None
        _check(lib().splitzip_decompress_batch_paged(self.items, self.n, self.dtype, C.byref(self.paging.c),
                                                     sizes.data_ptr() if sizes is not None else None, _stream_ptr(stream)),
               "splitzip_decompress_batch_paged")


# ---- a KV cache in pages: writing, reading, attention over it -----------------------------------------

def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


# what may hold a cache's words and rows, which are computed with: the type itself, or integers for bits
_WORDS = {BF16: (torch.bfloat16, torch.int16, torch.uint16), FP8_E5M2: (torch.float8_e5m2, torch.uint8, torch.int8),
          FP8_E4M3: (torch.float8_e4m3fn, torch.uint8, torch.int8), FP4_E2M1: (torch.float4_e2m1fn_x2, torch.uint8, torch.int8)}
_GROUP = 32   # 4-bit words that share a scale


_INT32, _INT64 = (torch.int32, torch.uint32), (torch.int64, torch.uint64)
_SCALES = (torch.uint8, torch.int8, torch.float8_e8m0fnu)   # the last one stands for just what a scale byte stands for


def _reached(*tensors) -> bool:
    """whether the GPU reaches the tensors (None: none): device memory, and pinned host memory"""
    return all(t is None or t.is_cuda or t.is_pinned() for t in tensors)


def _need_reached(*what) -> None:
    """for the general way, which takes an address as it is: descriptions (their tensors were looked at when they were made) and tensors"""
    for x in what:
        if not (_reached(x) if x is None or isinstance(x, torch.Tensor) else x._reached):
            raise ValueError("the tensors of a call, and those of its descriptions, must be on the GPU")


def _strides(t: torch.Tensor):
    """a tensor's strides, those of dimensions of one element as in a contiguous tensor (there they may be anything)"""
    out = list(t.stride())
    for k in range(t.dim() - 1, -1, -1):
        if t.shape[k] == 1:
            out[k] = t.shape[k + 1] * out[k + 1] if k + 1 < t.dim() else 1
    return tuple(out)


class KvCache:
    """splitzip_cache: K and V of one layer.

    k, v: device tensors [pages, page_tokens, kv_heads, head_dim] of the dtype's words (bfloat16, float8_e5m2 or float8_e4m3fn, or
    integers of that size), of the same strides, head_dim contiguous: views into a pool will do.  k_scales, v_scales (FP8): uint8 [pages, kv_heads, page_tokens]
    with contiguous pages.  FP4_E2M1: bytes of two words, the even element in the low half, [pages, page_tokens, kv_heads, head_dim / 2]
    (float4_e2m1fn_x2 or 8-bit integers), and scales uint8 [pages, kv_heads, head_dim / 32, page_tokens]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, dtype: int, k_scales: torch.Tensor | None = None,
                 v_scales: torch.Tensor | None = None):
        if k.dim() != 4 or k.shape != v.shape or _strides(k) != _strides(v) or k.stride(3) != 1:
            raise ValueError("k and v must be [pages, page_tokens, kv_heads, head_dim] with the same strides and a contiguous head_dim")
        es = _elem_size(dtype)
        if dtype not in _WORDS or k.dtype not in _WORDS[dtype] or v.dtype not in _WORDS[dtype]:
            raise ValueError("k and v must hold words of the dtype, as they are or as integers of their size")
        pages, tokens, heads, dim = k.shape
        scale_shape = (pages, heads, tokens)
        if dtype == FP4_E2M1:
            dim *= 2
            scale_shape = (pages, heads, dim // _GROUP, tokens)
        inner = [1]   # strides of a page's scales
        for n in scale_shape[:1:-1]:
            inner.insert(0, inner[0] * n)
        scale_stride = 0
        if dtype != BF16:
            if k_scales is None or v_scales is None:
                raise ValueError("an FP8 cache has scales" if dtype != FP4_E2M1 else "a cache of 4-bit words has scales")
            for s in (k_scales, v_scales):
                if (tuple(s.shape) != scale_shape or s.dtype not in _SCALES or _strides(s)[1:] != tuple(inner)
                        or _strides(s)[0] != _strides(k_scales)[0]):
                    raise ValueError(f"scales must be bytes [pages, kv_heads, {'' if dtype != FP4_E2M1 else 'head_dim / 32, '}page_tokens] with contiguous pages")
            scale_stride = _strides(k_scales)[0]
        self.dtype, self.kv_heads, self.head_dim = dtype, heads, dim
        self._keep = (k, v, k_scales, v_scales)
        self._reached = _reached(*self._keep)
        self.c = (_CCache if self._reached else _CCacheElsewhere)(k.data_ptr(), v.data_ptr(), _ptr(k_scales), _ptr(v_scales), dtype, heads, dim,
                         tokens, pages, 0, *(x * es for x in _strides(k)[:3]), scale_stride)

    @classmethod
    def zeros(cls, pages: int, page_tokens: int, kv_heads: int, head_dim: int, dtype: int, device="cuda") -> "KvCache":
        """A cache of its own memory, zeros."""
        row, groups = (head_dim // 2, (head_dim // _GROUP,)) if dtype == FP4_E2M1 else (head_dim, ())
        kv = [torch.zeros((pages, page_tokens, kv_heads, row), dtype=torch.bfloat16 if dtype == BF16 else torch.uint8, device=device) for _ in range(2)]
        scales = [None if dtype == BF16 else torch.zeros((pages, kv_heads, *groups, page_tokens), dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(*kv, dtype, *scales)

    @property
    def k(self) -> torch.Tensor:
        return self._keep[0]

    @property
    def v(self) -> torch.Tensor:
        return self._keep[1]

    @property
    def k_scales(self):
        return self._keep[2]

    @property
    def v_scales(self):
        return self._keep[3]


class KvCaches:
    """The marshalled list of a splitzip_cache_move call: caches of one geometry, the layers of a model."""

    def __init__(self, caches):
        self.n = len(caches)
        self._keep = list(caches)
        self._reached = all(c._reached for c in caches)
        self.items = (_CCache * max(self.n, 1))(*[c.c for c in caches]) if self._reached else None


class Sequences:
    """splitzip_seqs: the sequences of a call and its rows of each.

    block_table: int32 [n_seqs, pages of the longest] on the device (None: sequence s is page s); starts: int32 [n_seqs + 1],
    lens: int32 [n_seqs], on the device.  max_rows, max_len: the most rows of a sequence and the longest length, which the launches
    are cut for."""

    def __init__(self, block_table: torch.Tensor | None, starts: torch.Tensor, lens: torch.Tensor, max_rows: int, max_len: int):
        n = lens.numel()
        for t in (starts, lens):
            if t.dtype not in _INT32 or not t.is_contiguous():
                raise ValueError("starts and lens must be contiguous tensors of 32-bit integers")
        if starts.numel() != n + 1:
            raise ValueError("starts must have an entry more than lens")
        stride = 0
        if block_table is not None:
            if block_table.dim() != 2 or block_table.shape[0] != n or block_table.dtype not in _INT32 or not block_table.is_contiguous():
                raise ValueError("block_table must be a contiguous tensor [n_seqs, entries] of 32-bit page indices")
            stride = block_table.shape[1]
        self._keep = (block_table, starts, lens)
        self._reached = _reached(*self._keep)
        self.c = (_CSeqs if self._reached else _CSeqsElsewhere)(_ptr(block_table), starts.data_ptr(), lens.data_ptr(), stride, n, max_rows, max_len)


class Attention:
    """splitzip_attention: what a row sees and how its scores are shaped.

    slopes: float32 [q_heads]; tree: 64-bit words [n_rows, words], bit j of a row for row j of its sequence; positions: int32 [n_rows]
    (contiguous, on the device)."""

    def __init__(self, scale: float, softcap: float = 0.0, window: int = 0, slopes: torch.Tensor | None = None,
                 tree: torch.Tensor | None = None, positions: torch.Tensor | None = None):
        if slopes is not None and (slopes.dtype != torch.float32 or not slopes.is_contiguous()):
            raise ValueError("slopes must be contiguous float32")
        if tree is not None and (tree.dim() != 2 or tree.dtype not in _INT64 or not tree.is_contiguous()):
            raise ValueError("tree must be a contiguous tensor [n_rows, words] of 64-bit words")
        if positions is not None and (positions.dtype not in _INT32 or not positions.is_contiguous()):
            raise ValueError("positions must be a contiguous tensor of 32-bit integers")
        self._keep = (slopes, tree, positions)
        self._reached = _reached(*self._keep)
        self.c = (_CAttentionOf if self._reached else _CAttentionElsewhere)(scale, softcap, _ptr(slopes), _ptr(tree), _ptr(positions),
                               0 if tree is None else tree.shape[1], window, 0, *(-1 if t is None else t.shape[0] for t in self._keep))


class Rotation:
    """splitzip_rotation: norms of the heads of Q and K (with eps) and their rotation by position (with freqs).

    freqs: float32 [rotary_dim / 2], radians per position; q_weight, k_weight: [head_dim], both bfloat16 or both float32 (None: ones);
    positions: int32 [n_rows] (contiguous, on the device; None: a row's token's number)."""

    def __init__(self, freqs: torch.Tensor | None = None, interleaved: bool = False, scaling: float = 1.0, eps: float | None = None,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, weight_offset: float = 0.0,
                 positions: torch.Tensor | None = None):
        if freqs is not None and (freqs.dim() != 1 or freqs.dtype != torch.float32 or not freqs.is_contiguous()):
            raise ValueError("freqs must be contiguous float32 [rotary_dim / 2]")
        weights = [w for w in (q_weight, k_weight) if w is not None]
        if weights and eps is None:
            raise ValueError("weights are a norm's, which has an eps")
        if any(w.dim() != 1 or w.dtype not in (torch.bfloat16, torch.float32) or not w.is_contiguous() or w.shape != weights[0].shape
               or w.dtype != weights[0].dtype for w in weights):
            raise ValueError("weights must be contiguous [head_dim], both bfloat16 or both float32")
        if positions is not None and (positions.dim() != 1 or positions.dtype not in _INT32 or not positions.is_contiguous()):
            raise ValueError("positions must be a contiguous tensor [n_rows] of 32-bit integers")
        self._keep = (freqs, q_weight, k_weight, positions)
        self._reached = _reached(*self._keep)
        self.c = (_CRotationOf if self._reached else _CRotationElsewhere)(
            *(_ptr(t) for t in self._keep), scaling, 0.0 if eps is None else eps, weight_offset, 0 if freqs is None else 2 * freqs.shape[0],
            int(interleaved), int(eps is not None), int(bool(weights) and weights[0].dtype == torch.float32), 0,
            weights[0].shape[0] if weights else -1, -1 if positions is None else positions.shape[0])


class PagePool:
    """splitzip_pool: the pages that no sequence has.

    free: int32 [pages], the stack's entries; state: int32 [8], a splitzip_pool_state (POOL_STATE has its fields' names); both contiguous,
    on the device."""

    def __init__(self, free: torch.Tensor, state: torch.Tensor, page_tokens: int):
        for t in (free, state):
            if t.dim() != 1 or t.dtype not in _INT32 or not t.is_contiguous():
                raise ValueError("free and state must be contiguous tensors of 32-bit integers")
        if state.numel() != len(POOL_STATE):
            raise ValueError(f"state must have {len(POOL_STATE)} entries")
        if free.numel() >> 31 or page_tokens >> 31:
            raise ValueError("free must have less than 2^31 entries, page_tokens must be less and above 0")
        self._keep = (free, state)
        self._reached = _reached(*self._keep)
        self.c = (_CPool if self._reached else _CPoolElsewhere)(free.data_ptr(), state.data_ptr(), free.numel(), page_tokens, 0)

    @classmethod
    def full(cls, pages: int, page_tokens: int, device="cuda") -> "PagePool":
        """A pool that has all of its pages, page 0 on top."""
        state = torch.zeros(len(POOL_STATE), dtype=torch.int32, device=device)
        state[:1].fill_(pages)
        return cls(torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device), state, page_tokens)

    @property
    def free(self) -> torch.Tensor:
        return self._keep[0]

    @property
    def state(self) -> torch.Tensor:
        return self._keep[1]


POOL_STATE = ("free", "status", "lacking", "rows", "max_rows", "max_len", "taken", "given")


def read_pool_state(pool: PagePool) -> dict:
    """The pool's state on the host (waits for the device)."""
    return dict(zip(POOL_STATE, pool.state.tolist()))


def _rows(t: torch.Tensor, heads: int, dim: int, what: str) -> int:
    """words from row to row of a tensor [rows, heads, dim] of BF16 words"""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim or t.dtype not in _WORDS[BF16] or t.stride(2) != 1 or (heads > 1 and t.stride(1) != dim):
        raise ValueError(f"{what} must be [rows, {heads}, {dim}] of bfloat16 (or 16-bit integers) with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else heads * dim


def _write_or_read(name, cache: KvCache, seqs: Sequences, k: torch.Tensor, v: torch.Tensor, stream):
    f = getattr(lib(), name)
    ks, vs = _rows(k, cache.kv_heads, cache.head_dim, "k"), _rows(v, cache.kv_heads, cache.head_dim, "v")
    if k.shape[0] != v.shape[0]:
        raise ValueError("k and v must have the same number of rows")
    _need_reached(cache, seqs, k, v)
    _check(f(C.byref(cache.c), C.byref(seqs.c), k.data_ptr(), ks, v.data_ptr(), vs, k.shape[0], _stream_ptr(stream)), name)


def cache_write(k: torch.Tensor, v: torch.Tensor, cache: KvCache, seqs: Sequences, stream=None) -> None:
    """splitzip_cache_write: the BF16 rows k, v [rows, kv_heads, head_dim] become their sequences' last tokens, quantised if the cache is not BF16."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_write(cache.c, seqs.c, k, v, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_write") if rc else None
    _write_or_read("splitzip_cache_write", cache, seqs, k, v, stream)


def cache_read(cache: KvCache, seqs: Sequences, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """splitzip_cache_read: the rows' tokens out of the cache, as BF16, into k, v [rows, kv_heads, head_dim]."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_read(cache.c, seqs.c, k, v, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_read") if rc else None
    _write_or_read("splitzip_cache_read", cache, seqs, k, v, stream)


def cache_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, cache: KvCache, seqs: Sequences, how: Rotation,
                 q_out: torch.Tensor | None, k_out: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_cache_append: the BF16 rows k [rows, kv_heads, head_dim], normed and rotated, and v become their sequences' last tokens;
    q [rows, q_heads, head_dim] (None: none), normed and rotated, goes into q_out, which may be q itself, and k as BF16 into k_out."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_append(cache.c, seqs.c, how.c, q, q_out, k, v, k_out, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_append") if rc else None
    rows, heads, dim = k.shape[0], cache.kv_heads, cache.head_dim
    ks, vs = _rows(k, heads, dim, "k"), _rows(v, heads, dim, "v")
    kos = _rows(k_out, heads, dim, "k_out") if k_out is not None else 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if q is not None and q.dim() != 3:
        raise ValueError("q must be [rows, q_heads, head_dim]")
    q_heads = 0 if q is None else q.shape[1]
    qs, qos = (0, 0) if q is None else (_rows(q, q_heads, dim, "q"), _rows(q_out, q_heads, dim, "q_out"))
    if any(t is not None and t.shape[0] != rows for t in (q, q_out, v, k_out)):
        raise ValueError("q, q_out, k, v and k_out must have the same number of rows")
    if how.c.dim not in (-1, dim) or how.c.position_rows not in (-1, rows):
        raise ValueError(f"weights must have {dim} entries, positions {rows}")
    _need_reached(cache, seqs, how, q, q_out, k, v, k_out)
    _check(lib().splitzip_cache_append(C.byref(cache.c), C.byref(seqs.c), C.byref(how.c), _ptr(q), qs, _ptr(q_out), qos, k.data_ptr(), ks, v.data_ptr(), vs,
                                       _ptr(k_out), kos, rows, q_heads, _stream_ptr(stream)), "splitzip_cache_append")


def cache_allot(pool: PagePool, seqs: Sequences, rows: torch.Tensor, keep: torch.Tensor | None = None, slots: torch.Tensor | None = None,
                row_seqs: torch.Tensor | None = None, positions: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_cache_allot: sequence s keeps keep[s] tokens (None: all) and gets rows[s] more (int32 [n_seqs]); the block table, starts and
    lens that seqs was made of are written, and for each row of the step its slot (int64), sequence and position (int32; [n_rows] all, None: not
    wanted).  The pool's state says what became of it."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_allot(pool.c, seqs.c, rows, keep, slots, row_seqs, positions, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_allot") if rc else None
    for t, what in ((rows, "rows"), (keep, "keep")):
        if t is not None and (t.dim() != 1 or t.shape[0] != seqs.c.n_seqs or t.dtype not in _INT32 or not t.is_contiguous()):
            raise ValueError(f"{what} must be a contiguous tensor [n_seqs] of 32-bit integers")
    n_rows = {t.shape[0] for t in (slots, row_seqs, positions) if t is not None and t.dim() == 1}
    for t, types in ((slots, _INT64), (row_seqs, _INT32), (positions, _INT32)):
        if t is not None and (t.dim() != 1 or t.dtype not in types or not t.is_contiguous() or len(n_rows) != 1):
            raise ValueError("slots must be a contiguous tensor [n_rows] of 64-bit integers, row_seqs and positions as many of 32 bits")
    if any(n >> 32 for n in n_rows):   # (the library's word for them has 32 bits; from 2^30 on it refuses them)
        raise ValueError("slots, row_seqs and positions must have less than 2^32 entries")
    _need_reached(pool, seqs, rows, keep, slots, row_seqs, positions)
    _check(lib().splitzip_cache_allot(C.byref(pool.c), C.byref(seqs.c), rows.data_ptr(), _ptr(keep), _ptr(slots), _ptr(row_seqs), _ptr(positions),
                                      n_rows.pop() if n_rows else _MOST_ROWS, _stream_ptr(stream)), "splitzip_cache_allot")


def attention_workspace_bytes(cache: KvCache, seqs: Sequences, n_rows: int, q_heads: int) -> int:
    return int(lib().splitzip_attention_workspace_bytes(C.byref(cache.c), C.byref(seqs.c), n_rows, q_heads))


def attention_workspace(cache: KvCache, seqs: Sequences, n_rows: int, q_heads: int, device="cuda") -> torch.Tensor:
    """A workspace for cache_attention calls of up to n_rows rows over these sequences; one per stream."""
    return torch.empty(max(attention_workspace_bytes(cache, seqs, n_rows, q_heads), 16), dtype=torch.uint8, device=device)


def cache_attention(q: torch.Tensor, cache: KvCache, seqs: Sequences, out: torch.Tensor, workspace: torch.Tensor, how: Attention,
                    lse: torch.Tensor | None = None, stream=None) -> None:
    """splitzip_cache_attention: the BF16 rows q [rows, q_heads, head_dim] against their sequences' tokens, into out; lse float32 [rows, q_heads]."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_attention(cache.c, seqs.c, how.c, q, out, lse, workspace, None, None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_attention") if rc else None
    if q.dim() != 3:
        raise ValueError("q must be [rows, q_heads, head_dim]")
    rows, heads = q.shape[0], q.shape[1]
    qs, os_ = _rows(q, heads, cache.head_dim, "q"), _rows(out, heads, cache.head_dim, "out")
    if out.shape[0] != rows or (lse is not None and (tuple(lse.shape) != (rows, heads) or lse.dtype != torch.float32 or not lse.is_contiguous())):
        raise ValueError("out must have the rows of q, and lse be contiguous float32 [rows, q_heads]")
    for t, n, what in zip(how._keep, (heads, rows, rows), ("slopes", "tree", "positions")):
        if t is not None and t.shape[0] != n:
            raise ValueError(f"{what} must have {n} entries")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _need_reached(cache, seqs, how, q, out, lse, workspace)
    _check(lib().splitzip_cache_attention(C.byref(cache.c), C.byref(seqs.c), C.byref(how.c), q.data_ptr(), qs, out.data_ptr(), os_, _ptr(lse),
                                          rows, heads, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                          _stream_ptr(stream)), "splitzip_cache_attention")


def cache_move(caches: KvCaches, seqs: Sequences, path: torch.Tensor, n_rows: int | None = None, stream=None) -> None:
    """splitzip_cache_move: in all the caches, row path[s, i] of sequence s becomes its token base + i; path int32 [n_seqs, entries], -1 ends a
    path.  n_rows: rows of the call (all that starts says, if None)."""
    rc = (_lib or lib()).fast_cache.splitzip_cache_move(caches.items, caches.n, seqs.c, path, _MOST_ROWS if n_rows is None else n_rows,
                                                  None if stream is None else _handle(stream))
    if rc != _NOT_TAKEN:
        return _check(rc, "splitzip_cache_move") if rc else None
    if path.dim() != 2 or path.shape[0] != seqs.c.n_seqs or path.dtype not in _INT32 or not path.is_contiguous():
        raise ValueError("path must be a contiguous tensor [n_seqs, entries] of 32-bit integers")
    _need_reached(caches, seqs, path)
    _check(lib().splitzip_cache_move(caches.items, caches.n, C.byref(seqs.c), path.data_ptr(), path.shape[1],
                                     _MOST_ROWS if n_rows is None else n_rows, _stream_ptr(stream)), "splitzip_cache_move")


_MOST_ROWS = 1 << 30
