"""ctypes binding of include/wht_rotary.h (libwht_attention4.so): rotary positions of several axes, in training and in front of either cache.

Argument marshalling only, as in `attention`; a call on the current stream first goes to the extension module.  `autograd.wht_rotary` is
the same with a gradient.
"""
import operator

from . import attention4
from .attention import Rows, _empty, device_dummy
from .binding import DTYPE_BF16, DTYPE_F32, _DeviceGuard, _stream_handle, _torch

MAX_AXES = 4


class WhtRotaryError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({wht_rotary_status_string(status)})")


def wht_rotary_status_string(status: int) -> str:
    return attention4.library().wht_rotary_status_string(int(status)).decode()


def wht_rotary_axes(sections, cyclic=False) -> bytes:
    """The axis of every pair: sections[a] pairs of axis a, one axis after the other, or (cyclic) the axes in turn for as long as each has some left."""
    left = [int(n) for n in sections]
    if not 1 <= len(left) <= MAX_AXES or min(left) < 0:
        raise ValueError(f"sections must be 1 to {MAX_AXES} numbers of pairs, got {list(sections)}")
    if not cyclic:
        return bytes(a for a, n in enumerate(left) for _ in range(n))
    out = []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return bytes(out)


def _axis_bytes(axes):
    """axes as bytes, number by number: bytes() of a number is so many zeros, of an array its memory."""
    if axes is None or type(axes) is bytes:
        return axes
    try:
        return bytes([operator.index(a) for a in axes])
    except (TypeError, ValueError):
        raise TypeError("axes must be the axis of each pair: bytes, or small whole numbers") from None


def _axes(axes, rotary, count):
    """The bytes that the library reads: one for each pair, below `count`."""
    axes = _axis_bytes(axes)
    if axes is None:
        return None
    if len(axes) != rotary // 2:
        raise ValueError(f"axes must have one number for each of the {rotary // 2} pairs, got {len(axes)}")
    if axes and max(axes) >= count:
        raise ValueError(f"axes must be below {count}, the number of positions a token has, got {max(axes)}")
    return axes


def _rope(rope, device, torch):
    """(address, rows, rotary) of a table of cos and sin."""
    if not rope.is_cuda or rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[2] != 2 or not rope.is_contiguous() or rope.device != device:
        raise ValueError("rope must be a contiguous float32 [positions, rotary / 2, 2] tensor on the tensors' device")
    return rope.data_ptr() or device_dummy(torch, device), rope.shape[0], 2 * rope.shape[1]


def _positions(positions, T, device, torch):
    """(address, axes) of positions [T, axes], or [T] for one axis."""
    if positions is None:
        return None, 1
    if positions.dim() not in (1, 2) or positions.shape[0] != T or not positions.is_cuda or positions.dtype != torch.int32 or not positions.is_contiguous() \
            or positions.device != device or (positions.dim() == 2 and not 1 <= positions.shape[1] <= MAX_AXES):
        raise ValueError(f"positions must be a contiguous int32 [{T}] or [{T}, axes] tensor on the tensors' device, of up to {MAX_AXES} axes")
    return positions.data_ptr() or device_dummy(torch, device), 1 if positions.dim() == 1 else positions.shape[1]


def wht_rotary_rotate(x, rope, positions=None, axes=None, interleaved=False, inverse=False, out=None, stream=None):
    """x with the first 2 * rope.shape[1] elements of every head turned, pair by pair, by the angle of the token's position on the pair's axis.
      x [T, heads, head_dim]: bfloat16 | float32, any strides with 16-byte steps
      rope [positions, rotary / 2, 2] float32 (wht_attention_rope_table)
      positions int32 [T, axes] or [T] (None: token t has position t)
      axes: the axis of each pair, bytes or whole numbers (wht_rotary_axes; None: all on the first)
      inverse: turn back, which is also the gradient; out: may be x
    """
    if stream is None:
        done = attention4._native().rotate(x, rope, positions, axes, interleaved, inverse, out)
        if done is not None:
            if type(done) is int:
                raise WhtRotaryError(done, "wht_rotary_rotate")
            return done
    torch = _torch()
    if not x.is_cuda or x.dim() != 3 or (x.shape[2] > 1 and x.stride(2) != 1):
        raise ValueError("x must be a [T, heads, head_dim] GPU tensor with a contiguous last dimension")
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"tensors must be float32 or bfloat16, got {x.dtype}")
    T, heads, head_dim = x.shape
    attention4._whole(heads, "heads")
    attention4._whole(head_dim, "head_dim")
    rope_at, rope_rows, rotary = _rope(rope, x.device, torch)
    positions_at, count = _positions(positions, T, x.device, torch)
    axes = _axes(axes, rotary, count)
    if out is None:
        out = _empty(x.shape, x.dtype, x.device, stream, torch)
    elif out.shape != x.shape or out.dtype != x.dtype or out.device != x.device or (head_dim > 1 and out.stride(2) != 1):
        raise ValueError("out must match x in shape, dtype and device, with a contiguous last dimension")
    if T == 0:
        return out
    with _DeviceGuard(torch, x.device):
        rc = attention4.library().wht_rotary_rotate(
            Rows(x.data_ptr(), x.stride(0), x.stride(1)), Rows(out.data_ptr(), out.stride(0), out.stride(1)), T, heads, head_dim, rope_at, rope_rows, rotary,
            int(bool(interleaved)), positions_at, count, axes, int(bool(inverse)), DTYPE_F32 if x.dtype == torch.float32 else DTYPE_BF16,
            _stream_handle(stream, torch, x.device))
    if rc != 0:
        raise WhtRotaryError(rc, "wht_rotary_rotate")
    return out
