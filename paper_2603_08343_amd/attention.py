"""ctypes binding of libwht_attention.so -- same names as the C ABI (include/wht_attention.h): the paged cache and the
attention whose concatenated head outputs the Walsh-Hadamard output layer takes.

Argument marshalling only, as in `binding`: torch supplies device memory and the stream, every step runs in the HIP kernels; wrong
arguments raise TypeError or ValueError, a status of the library WhtAttentionError.  A call on the current stream first goes to the
extension module _attention_marshal (csrc/attention_marshal.cpp), which does the same in native code and hands back None for
anything but a plain valid call; the code here then decides, and words the errors.
"""
import ctypes
import math
import os
import warnings

from .binding import DTYPE_BF16, DTYPE_F32, _DeviceGuard, _stream_handle, _torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libwht_attention.so")
_lib = None

EXPORTS = ("wht_attention_append", "wht_attention_workspace_bytes", "wht_attention_paged", "wht_attention_status_string")


class WhtAttentionError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({wht_attention_status_string(status)})")


class Rows(ctypes.Structure):
    """wht_attention_rows_t"""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Cache(ctypes.Structure):
    """wht_attention_cache_t"""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("pages", ctypes.c_int32), ("heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class Batch(ctypes.Structure):
    """wht_attention_batch_t"""
    _fields_ = [("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("q_starts", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("B", ctypes.c_int32), ("width", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def library():
    """The loaded shared library.  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2603_08343_amd.build` "
                               "(hipcc, gfx950). The attention has no CPU or eager fallback.")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i64, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
        rows, cache, batch = ctypes.POINTER(Rows), ctypes.POINTER(Cache), ctypes.POINTER(Batch)
        lib.wht_attention_append.argtypes = [rows, rows, rows, rows, i64, i32, cache, batch, vp, i64, i32, i32, i64, i32, vp]
        lib.wht_attention_append.restype = ctypes.c_int
        lib.wht_attention_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, i64, i64, i32]
        lib.wht_attention_workspace_bytes.restype = sz
        lib.wht_attention_paged.argtypes = [rows, rows, vp, i64, i32, cache, batch, vp, i64, i32, i64, f32, i32, vp, sz, vp]
        lib.wht_attention_paged.restype = ctypes.c_int
        lib.wht_attention_status_string.argtypes = [ctypes.c_int]
        lib.wht_attention_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def wht_attention_status_string(status: int) -> str:
    return library().wht_attention_status_string(int(status)).decode()


def _whole(x, name, bits=32):
    """x as an int that the library's argument of so many bits holds; ctypes would cut off what does not fit."""
    try:
        n = int(x)
    except (TypeError, ValueError, OverflowError):
        raise TypeError(f"{name} must be a whole number, got {x!r}") from None
    if n != x or not -(1 << (bits - 1)) <= n < 1 << (bits - 1):
        raise ValueError(f"{name} must be a whole number of {bits} bits, got {x!r}")
    return n


def wht_attention_workspace_bytes(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length, dtype) -> int:
    return int(library().wht_attention_workspace_bytes(
        _whole(T, "T", 64), _whole(B, "B"), _whole(q_heads, "q_heads"), _whole(heads, "heads"), _whole(head_dim, "head_dim"), _whole(max_q, "max_q"),
        _whole(max_length, "max_length", 64), _whole(prefix_length, "prefix_length", 64), _whole(dtype, "dtype")))


def wht_attention_rope_table(positions, rotary, base=10000.0, device="cuda"):
    """[positions, rotary / 2, 2] float32: cos and sin of position * base^(-2 i / rotary), from angles in 64 bits."""
    import torch
    if rotary < 0 or rotary % 2 != 0:
        raise ValueError(f"rotary must be even and not negative, got {rotary}")
    rates = base ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device=device) / rotary)
    angles = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * rates
    return torch.stack((angles.cos(), angles.sin()), dim=2).float()


# ------------------------------------------------------------------ tensor calls

def _code(t, torch):
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_F32
    raise TypeError(f"tensors must be float32 or bfloat16, got {t.dtype}")


def _rows(t, name, like, heads=None):
    """A [T, heads, head_dim] tensor as the library takes it; `like`: the cache's pages."""
    if not t.is_cuda or t.dim() != 3 or t.shape[2] != like.shape[3] or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be a [T, heads, {like.shape[3]}] GPU tensor with a contiguous last dimension")
    if t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name} must have the cache's dtype and device")
    if heads is not None and t.shape[1] != heads:
        raise ValueError(f"{name} must have {heads} heads, got {t.shape[1]}")
    return Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _cache(k_pages, v_pages):
    if k_pages.dim() != 4 or not k_pages.is_cuda or k_pages.stride(3) != 1:
        raise ValueError("k_pages must be a [pages, heads, page_size, head_dim] GPU tensor with a contiguous last dimension")
    if 0 in k_pages.shape:
        raise ValueError(f"k_pages must not be empty, got {list(k_pages.shape)}")
    if v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype or v_pages.device != k_pages.device or v_pages.stride() != k_pages.stride():
        raise ValueError("v_pages must match k_pages in shape, strides, dtype and device")
    pages, heads, page_size, head_dim = k_pages.shape
    ps, hs, ts, _ = k_pages.stride()
    for n, name in ((pages, "the number of pages"), (heads, "heads"), (page_size, "page_size"), (head_dim, "head_dim")):
        _whole(n, name)
    return Cache(k_pages.data_ptr(), v_pages.data_ptr(), ps, hs, ts, pages, heads, page_size, head_dim)


def _ints(t, name, shape, device, torch):
    if not t.is_cuda or t.dtype != torch.int32 or tuple(t.shape) != shape or t.device != device or (len(shape) == 1 and not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous int32 {list(shape)} tensor on the cache's device")
    return t.data_ptr()


def _batch(table, lengths, q_starts, T, device, torch):
    if table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be an int32 [B, width] tensor with contiguous rows")
    B, width = table.shape
    _whole(B, "the number of sequences")
    _whole(width, "the table's width")
    _ints(table, "table", (B, width), device, torch)
    _ints(lengths, "lengths", (B,), device, torch)
    if q_starts is not None:
        _ints(q_starts, "q_starts", (B + 1,), device, torch)
    elif T != B:
        raise ValueError(f"without q_starts every sequence has one row: {B} sequences, {T} rows")
    # torch gives an empty tensor a NULL address; the library reads none of these where B = 0
    at = table.data_ptr() or device_dummy(torch, device)
    return Batch(at, lengths.data_ptr() or at, None if q_starts is None else q_starts.data_ptr(), table.stride(0), B, width)


def _empty(shape, dtype, device, stream, torch):
    """Memory for a call on `stream`, of that stream's own: what the current stream last freed may still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


_dummies = {}


def device_dummy(torch, device):
    if device not in _dummies:
        _dummies[device] = torch.zeros(64, dtype=torch.int32, device=device)
    return _dummies[device].data_ptr()


_native_module = None


class _NoNative:
    """Stands in for the extension module where it cannot be used: declines every call."""
    append = paged = staticmethod(lambda *args: None)


def _load_native(torch, lib):
    current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    try:
        from . import _attention_marshal
        built_for = getattr(_attention_marshal, "torch_version", "unknown")
        if current_stream is None or built_for != str(torch.__version__):
            raise ImportError(f"built for torch {built_for}, this is {torch.__version__}")
    except ImportError as e:
        warnings.warn(f"the extension module _attention_marshal cannot be used ({e}): tensor calls take about 10 us longer "
                      "each; build it with `python -m paper_2603_08343_amd.build`", RuntimeWarning, stacklevel=4)
        return _NoNative
    names = ("wht_attention_append", "wht_attention_workspace_bytes", "wht_attention_paged")
    _attention_marshal.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names), current_stream)
    return _attention_marshal


def _native():
    """The extension module, loaded and told the library's addresses on the first tensor call."""
    global _native_module
    if _native_module is None:
        _native_module = _load_native(_torch(), library())
    return _native_module


def wht_attention_append(q, k, v, k_pages, v_pages, table, lengths, rope, q_starts=None, position=0, interleaved=False, q_out=None,
                         stream=None):
    """Append a batch's new tokens to the paged cache: k (rotated) and v go to their places in k_pages and v_pages, and the
    rotated q is returned (None where q is None).
      q [T, q_heads, head_dim], k, v [T, heads, head_dim]: bfloat16 | float32, any strides with 16-byte steps
      k_pages, v_pages [pages, heads, page_size, head_dim]: any order in memory (equal strides)
      table int32 [B, width], lengths int32 [B] (the new tokens included), q_starts int32 [B + 1] (None: a token each)
      rope [positions, rotary / 2, 2] float32 (wht_attention_rope_table) or None; position: of a sequence's first own token
    For serving: nothing here is recorded for a backward pass.
    """
    if stream is None:
        done = _native().append(q, k, v, k_pages, v_pages, table, lengths, rope, q_starts, position, interleaved, q_out)
        if done is not None:
            if type(done) is int:
                raise WhtAttentionError(done, "wht_attention_append")
            return None if q is None else done
    torch = _torch()
    cache = _cache(k_pages, v_pages)
    code = _code(k_pages, torch)
    T, heads = k.shape[0], k_pages.shape[1]
    kr, vr = _rows(k, "k", k_pages, heads), _rows(v, "v", k_pages, heads)
    if v.shape[0] != T:
        raise ValueError("k and v must have the same number of rows")
    qr, outr, q_heads = Rows(None, 0, 0), Rows(None, 0, 0), 0
    if q is None:
        q_out = None
    else:
        qr, q_heads = _rows(q, "q", k_pages), _whole(q.shape[1], "q_heads")
        if q.shape[0] != T:
            raise ValueError("q and k must have the same number of rows")
        if q_out is None:
            q_out = _empty(q.shape, q.dtype, q.device, stream, torch)
        outr = _rows(q_out, "q_out", k_pages, q_heads)
        if q_out.shape[0] != T:
            raise ValueError("q_out and q must have the same number of rows")
    batch = _batch(table, lengths, q_starts, T, k_pages.device, torch)
    rope_at, rope_rows, rotary = None, 0, 0
    if rope is not None:
        if not rope.is_cuda or rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[2] != 2 or not rope.is_contiguous() \
                or rope.device != k_pages.device:
            raise ValueError("rope must be a contiguous float32 [positions, rotary / 2, 2] tensor on the cache's device")
        rope_rows, rotary = rope.shape[0], _whole(2 * rope.shape[1], "rotary")
        rope_at = rope.data_ptr() or device_dummy(torch, rope.device)
    position = _whole(position, "position", 64)
    if T == 0:
        return q_out
    with _DeviceGuard(torch, k_pages.device):
        rc = library().wht_attention_append(qr, kr, vr, outr, T, q_heads, cache, batch, rope_at, rope_rows, rotary, int(bool(interleaved)),
                                            position, code, _stream_handle(stream, torch, k_pages.device))
    if rc != 0:
        raise WhtAttentionError(rc, "wht_attention_append")
    return q_out


def wht_attention_paged(q, k_pages, v_pages, table, lengths, q_starts=None, prefix_table=None, prefix_length=0, max_q=None, max_length=None,
                        scale=None, out=None, lse=None, want_lse=False, workspace=None, stream=None):
    """Softmax attention of a batch's new tokens over the paged cache: every token sees the shared prefix and its own sequence up to itself.
    Returns out [T, q_heads, head_dim], or (out, lse [T, q_heads] float32) with want_lse or a given lse.
      q [T, q_heads, head_dim]: q_heads a multiple of the cache's heads
      prefix_table int32 [>= ceil(prefix_length / page_size)]
      max_q: at least the largest number of new tokens of a sequence (None: 1 without q_starts, T with them)
      max_length: at least the largest of lengths (None: what the table can hold); goes into how the work is split
      scale: None for 1 / sqrt(head_dim)
    For serving: nothing here is recorded for a backward pass.
    """
    if stream is None:
        done = _native().paged(q, k_pages, v_pages, table, lengths, q_starts, prefix_table, prefix_length, max_q, max_length, scale, out, lse,
                               want_lse, workspace)
        if done is not None:
            if type(done) is int:
                raise WhtAttentionError(done, "wht_attention_paged")
            return done
    torch = _torch()
    cache = _cache(k_pages, v_pages)
    code = _code(k_pages, torch)
    qr = _rows(q, "q", k_pages)
    T, q_heads, head_dim = q.shape
    _whole(q_heads, "q_heads")
    batch = _batch(table, lengths, q_starts, T, k_pages.device, torch)
    if out is None:
        out = _empty((T, q_heads, head_dim), q.dtype, q.device, stream, torch)
    outr = _rows(out, "out", k_pages, q_heads)
    if out.shape[0] != T:
        raise ValueError("out and q must have the same number of rows")
    if lse is not None:
        if not lse.is_cuda or lse.dtype != torch.float32 or lse.shape != (T, q_heads) or not lse.is_contiguous() or lse.device != q.device:
            raise ValueError("lse must be a contiguous float32 [T, q_heads] tensor on q's device")
    elif want_lse:
        lse = _empty((T, q_heads), torch.float32, q.device, stream, torch)
    prefix_length = _whole(prefix_length, "prefix_length", 64)
    if prefix_length > 0:
        need = -(-prefix_length // k_pages.shape[2])
        if prefix_table is None or prefix_table.dim() != 1 or prefix_table.numel() < need:
            raise ValueError(f"prefix_table must name the {need} pages of prefix_length = {prefix_length}")
        _ints(prefix_table, "prefix_table", tuple(prefix_table.shape), k_pages.device, torch)
    max_q = _whole(max_q, "max_q") if max_q is not None else 1 if q_starts is None else max(T, 1)
    max_length = _whole(max_length, "max_length", 64) if max_length is not None else table.shape[1] * k_pages.shape[2]
    if scale is None:
        scale = 1.0 / math.sqrt(head_dim)
    if T > 0:
        need = wht_attention_workspace_bytes(T, table.shape[0], q_heads, k_pages.shape[1], head_dim, max_q, max_length, prefix_length, code)
        if workspace is None:
            workspace = _empty(need, torch.uint8, q.device, stream, torch) if need else None
        elif not workspace.is_cuda or not workspace.is_contiguous() or workspace.device != q.device:
            raise ValueError("workspace must be a contiguous GPU tensor on q's device")
        with _DeviceGuard(torch, q.device):
            rc = library().wht_attention_paged(qr, outr, None if lse is None else lse.data_ptr(), T, q_heads, cache, batch,
                                               prefix_table.data_ptr() if prefix_length > 0 else None, prefix_length, max_q, max_length,
                                               float(scale), code, None if workspace is None else workspace.data_ptr(),
                                               0 if workspace is None else workspace.numel() * workspace.element_size(),
                                               _stream_handle(stream, torch, q.device))
        if rc != 0:
            raise WhtAttentionError(rc, "wht_attention_paged")
    return out if lse is None else (out, lse)
