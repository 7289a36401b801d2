"""ctypes binding of libwht_attention4.so -- same names as the C ABI (include/wht_attention4.h): the paged cache in 4 bits and its attention.

Argument marshalling only, as in `attention`: torch supplies device memory and the stream, every step runs in the HIP kernels; wrong
arguments raise TypeError or ValueError, a status of the library WhtAttention4Error.  A call on the current stream first goes to the
extension module _attention_marshal (csrc/attention_marshal.cpp), which hands back None for anything but a plain valid call; the code here
then decides, and words the errors.
"""
import ctypes
import math
import os

from . import attention
from .attention import Batch, Rows, _batch, _empty, _ints, _whole
from .binding import DTYPE_BF16, DTYPE_F32, _DeviceGuard, _stream_handle, _torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libwht_attention4.so")
_lib = None

EXPORTS = ("wht_attention_append4", "wht_attention4_workspace_bytes", "wht_attention_paged4", "wht_attention4_status_string")
ROTARY_EXPORTS = ("wht_rotary_rotate", "wht_rotary_status_string")


class WhtAttention4Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({wht_attention4_status_string(status)})")


class Cache4(ctypes.Structure):
    """wht_attention_cache4_t"""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64), ("scale_token_stride", ctypes.c_int64),
                ("pages", ctypes.c_int32), ("heads", ctypes.c_int32), ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


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
        rows, cache, batch = ctypes.POINTER(Rows), ctypes.POINTER(Cache4), ctypes.POINTER(Batch)
        lib.wht_attention_append4.argtypes = [rows, rows, rows, rows, rows, rows, i64, i32, cache, batch, vp, i64, i32, i32, i64, vp, i32, ctypes.c_char_p,
                                              i32, i32, vp]
        lib.wht_attention_append4.restype = ctypes.c_int
        lib.wht_attention4_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, i64, i64, i32]
        lib.wht_attention4_workspace_bytes.restype = sz
        lib.wht_attention_paged4.argtypes = [rows, rows, vp, i64, i32, cache, batch, vp, i64, i32, i64, f32, i32, i32, vp, sz, vp]
        lib.wht_attention_paged4.restype = ctypes.c_int
        lib.wht_rotary_rotate.argtypes = [rows, rows, i64, i32, i32, vp, i64, i32, i32, vp, i32, ctypes.c_char_p, i32, i32, vp]
        lib.wht_rotary_rotate.restype = ctypes.c_int
        for name in ("wht_attention4_status_string", "wht_rotary_status_string"):
            getattr(lib, name).argtypes = [ctypes.c_int]
            getattr(lib, name).restype = ctypes.c_char_p
        _lib = lib
    return _lib


def wht_attention4_status_string(status: int) -> str:
    return library().wht_attention4_status_string(int(status)).decode()


def wht_attention4_workspace_bytes(T, B, q_heads, heads, head_dim, max_q, max_length, prefix_length, dtype) -> int:
    return int(library().wht_attention4_workspace_bytes(
        _whole(T, "T", 64), _whole(B, "B"), _whole(q_heads, "q_heads"), _whole(heads, "heads"), _whole(head_dim, "head_dim"), _whole(max_q, "max_q"),
        _whole(max_length, "max_length", 64), _whole(prefix_length, "prefix_length", 64), _whole(dtype, "dtype")))


_native_module = None


class _NoNative:
    """Stands in for the extension module where it cannot be used: declines every call."""
    append4 = paged4 = rotate = rotary = staticmethod(lambda *args: None)
    leaf_elsewhere = staticmethod(lambda x: False)


def _native():
    """The extension module, told this library's addresses on the first tensor call."""
    global _native_module
    if _native_module is None:
        module, lib = attention._native(), library()
        if module is attention._NoNative:
            _native_module = _NoNative
        else:
            names = ("wht_attention_append4", "wht_attention4_workspace_bytes", "wht_attention_paged4", "wht_rotary_rotate")
            from .autograd import WhtRotaryFunction
            module.bind4(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names), WhtRotaryFunction.apply)
            _native_module = module
    return _native_module


# ------------------------------------------------------------------ tensor calls

def _cache4(k_pages, v_pages, k_scales, v_scales, torch):
    if k_pages.dim() != 4 or not k_pages.is_cuda or k_pages.dtype != torch.uint8 or k_pages.stride(3) != 1:
        raise ValueError("k_pages must be a uint8 [pages, heads, page_size, head_dim / 2] GPU tensor with a contiguous last dimension")
    if 0 in k_pages.shape:
        raise ValueError(f"k_pages must not be empty, got {list(k_pages.shape)}")
    if v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype or v_pages.device != k_pages.device or v_pages.stride() != k_pages.stride():
        raise ValueError("v_pages must match k_pages in shape, strides, dtype and device")
    pages, heads, page_size, half = k_pages.shape
    if half % 16 != 0:
        raise ValueError(f"k_pages must hold heads of a multiple of 32 elements, got {2 * half}")
    if tuple(k_scales.shape) != (pages, heads, page_size, half // 16) or k_scales.dtype != torch.uint8 or k_scales.device != k_pages.device \
            or (half > 16 and k_scales.stride(3) != 1):
        raise ValueError(f"k_scales must be a uint8 {[pages, heads, page_size, half // 16]} tensor on k_pages' device with a contiguous last dimension")
    if v_scales.shape != k_scales.shape or v_scales.dtype != k_scales.dtype or v_scales.device != k_scales.device or v_scales.stride() != k_scales.stride():
        raise ValueError("v_scales must match k_scales in shape, strides, dtype and device")
    for n, name in ((pages, "the number of pages"), (heads, "heads"), (page_size, "page_size"), (2 * half, "head_dim")):
        _whole(n, name)
    return Cache4(k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), *k_pages.stride()[:3], *k_scales.stride()[:3],
                  pages, heads, page_size, 2 * half)


def _rows4(t, name, like, pages, torch, heads=None):
    """A [T, heads, head_dim] tensor as the library takes it, of the type of `like`."""
    head_dim = 2 * pages.shape[3]
    if not t.is_cuda or t.dim() != 3 or t.shape[2] != head_dim or t.stride(2) != 1:
        raise ValueError(f"{name} must be a [T, heads, {head_dim}] GPU tensor with a contiguous last dimension")
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"tensors must be float32 or bfloat16, got {t.dtype}")
    if t.dtype != like.dtype or t.device != pages.device:
        raise ValueError(f"{name} must have the other tensors' dtype and the cache's device")
    if heads is not None and t.shape[1] != heads:
        raise ValueError(f"{name} must have {heads} heads, got {t.shape[1]}")
    return Rows(t.data_ptr(), t.stride(0), t.stride(1))


def wht_attention_append4(q, k, v, k_pages, v_pages, k_scales, v_scales, table, lengths, rope, q_starts=None, position=0, positions=None, axes=None,
                          interleaved=False, transform=True, q_out=None, k_out=None, v_out=None, want_values=False, stream=None):
    """Append a batch's new tokens to the paged cache in 4 bits: k (rotated, transformed) and v (transformed) go to their places as codes and
    scales, and the rotated and transformed q is returned (None where q is None); with want_values, or given k_out and v_out, (q, k_out, v_out):
    the numbers that the stored codes stand for.
      q [T, q_heads, head_dim], k, v [T, heads, head_dim]: bfloat16 | float32, any strides with 16-byte steps
      k_pages, v_pages uint8 [pages, heads, page_size, head_dim / 2], k_scales, v_scales uint8 [pages, heads, page_size, head_dim / 32]
      table int32 [B, width], lengths int32 [B] (the new tokens included), q_starts int32 [B + 1] (None: a token each)
      rope [positions, rotary / 2, 2] float32 (wht_attention_rope_table) or None; position: of a sequence's first own token
      positions int32 [T, axes] and axes (wht_rotary_axes): positions of several axes, in place of a token's own
      transform: every 32 elements pass a Walsh-Hadamard transform; wht_attention_paged4 takes it back
    For serving: nothing here is recorded for a backward pass.
    """
    if stream is None:
        done = _native().append4(q, k, v, k_pages, v_pages, k_scales, v_scales, table, lengths, rope, q_starts, position, positions, axes, interleaved,
                                 transform, q_out, k_out, v_out, want_values)
        if done is not None:
            if type(done) is int:
                raise WhtAttention4Error(done, "wht_attention_append4")
            return None if type(done) is tuple and not done else done
    from . import rotary as _rotary
    torch = _torch()
    cache = _cache4(k_pages, v_pages, k_scales, v_scales, torch)
    T, heads = k.shape[0], k_pages.shape[1]
    kr, vr = _rows4(k, "k", k, k_pages, torch, heads), _rows4(v, "v", k, k_pages, torch, heads)
    if v.shape[0] != T:
        raise ValueError("k and v must have the same number of rows")
    if (k_out is None) != (v_out is None):
        raise ValueError("k_out and v_out come together")
    none = Rows(None, 0, 0)
    qr, outr, kor, vor, q_heads = none, none, none, none, 0
    if q is None:
        q_out = None
    else:
        qr, q_heads = _rows4(q, "q", k, k_pages, torch), _whole(q.shape[1], "q_heads")
        if q.shape[0] != T:
            raise ValueError("q and k must have the same number of rows")
        if q_out is None:
            q_out = _empty(q.shape, q.dtype, q.device, stream, torch)
        outr = _rows4(q_out, "q_out", k, k_pages, torch, q_heads)
        if q_out.shape[0] != T:
            raise ValueError("q_out and q must have the same number of rows")
    if want_values or k_out is not None:
        if k_out is None:
            k_out, v_out = (_empty(k.shape, k.dtype, k.device, stream, torch) for _ in range(2))
        kor, vor = _rows4(k_out, "k_out", k, k_pages, torch, heads), _rows4(v_out, "v_out", k, k_pages, torch, heads)
        if k_out.shape[0] != T or v_out.shape[0] != T:
            raise ValueError("k_out, v_out and k must have the same number of rows")
    batch = _batch(table, lengths, q_starts, T, k_pages.device, torch)
    rope_at, rope_rows, rotary = (None, 0, 0) if rope is None else _rotary._rope(rope, k_pages.device, torch)
    positions_at, count = _rotary._positions(positions, T, k_pages.device, torch)
    axes = _rotary._axes(axes, rotary, count)
    position = _whole(position, "position", 64)
    if T > 0:
        with _DeviceGuard(torch, k_pages.device):
            rc = library().wht_attention_append4(qr, kr, vr, outr, kor, vor, T, q_heads, cache, batch, rope_at, rope_rows, rotary, int(bool(interleaved)),
                                                 position, positions_at, count, axes, int(bool(transform)),
                                                 DTYPE_F32 if k.dtype == torch.float32 else DTYPE_BF16, _stream_handle(stream, torch, k_pages.device))
        if rc != 0:
            raise WhtAttention4Error(rc, "wht_attention_append4")
    return q_out if k_out is None else (q_out, k_out, v_out)


def wht_attention_paged4(q, k_pages, v_pages, k_scales, v_scales, table, lengths, q_starts=None, prefix_table=None, prefix_length=0, max_q=None,
                         max_length=None, scale=None, transform=True, out=None, lse=None, want_lse=False, workspace=None, stream=None):
    """Softmax attention of a batch's new tokens over the paged cache in 4 bits: every token sees the shared prefix and its own sequence up to itself.
    Returns out [T, q_heads, head_dim], or (out, lse [T, q_heads] float32) with want_lse or a given lse.
      q [T, q_heads, head_dim]: bfloat16 | float32, q_heads a multiple of the cache's heads; as wht_attention_append4 returned it
      prefix_table int32 [>= ceil(prefix_length / page_size)]
      max_q: at least the largest number of new tokens of a sequence (None: 1 without q_starts, T with them)
      max_length: at least the largest of lengths (None: what the table can hold); goes into how the work is split
      scale: None for 1 / sqrt(head_dim);  transform: as the tokens were appended
      workspace: wht_attention4_workspace_bytes of this call's sizes (None: allocated); a larger batch may need fewer
    For serving: nothing here is recorded for a backward pass.
    """
    if stream is None:
        done = _native().paged4(q, k_pages, v_pages, k_scales, v_scales, table, lengths, q_starts, prefix_table, prefix_length, max_q, max_length, scale,
                                transform, out, lse, want_lse, workspace)
        if done is not None:
            if type(done) is int:
                raise WhtAttention4Error(done, "wht_attention_paged4")
            return done
    torch = _torch()
    cache = _cache4(k_pages, v_pages, k_scales, v_scales, torch)
    qr = _rows4(q, "q", q, k_pages, torch)
    T, q_heads, head_dim = q.shape
    code = DTYPE_F32 if q.dtype == torch.float32 else DTYPE_BF16
    _whole(q_heads, "q_heads")
    batch = _batch(table, lengths, q_starts, T, k_pages.device, torch)
    if out is None:
        out = _empty((T, q_heads, head_dim), q.dtype, q.device, stream, torch)
    outr = _rows4(out, "out", q, k_pages, torch, q_heads)
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
        need = wht_attention4_workspace_bytes(T, table.shape[0], q_heads, k_pages.shape[1], head_dim, max_q, max_length, prefix_length, code)
        if workspace is None:
            workspace = _empty(need, torch.uint8, q.device, stream, torch) if need else None
        elif not workspace.is_cuda or not workspace.is_contiguous() or workspace.device != q.device:
            raise ValueError("workspace must be a contiguous GPU tensor on q's device")
        with _DeviceGuard(torch, q.device):
            rc = library().wht_attention_paged4(qr, outr, None if lse is None else lse.data_ptr(), T, q_heads, cache, batch,
                                                prefix_table.data_ptr() if prefix_length > 0 else None, prefix_length, max_q, max_length,
                                                float(scale), int(bool(transform)), code, None if workspace is None else workspace.data_ptr(),
                                                0 if workspace is None else workspace.numel() * workspace.element_size(),
                                                _stream_handle(stream, torch, q.device))
        if rc != 0:
            raise WhtAttention4Error(rc, "wht_attention_paged4")
    return out if lse is None else (out, lse)
