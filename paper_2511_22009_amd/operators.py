"""Operators on torch tensors that need no model: 8-bit row quantisation and products,
rotary positions with several axes, and the norm of queries and keys with the rotation
(the calls without a model in include/streamflow.h, which states their formulas).

As in the rest of the binding, tensors give device memory and streams, and shapes, types
and devices are checked before a call: TypeError for what is no fitting tensor, ValueError
for sizes and strides, SFError for what the library refuses. A call runs on the device of
its tensors, on `stream` or torch's current stream there. Outputs that are not given are
allocated for that stream. With a `stream` other than the current one, ordering it after
the work that fills the inputs is the caller's, as in torch; the inputs' memory is kept
until the stream is done with it. Nothing is differentiated: a tensor that requires grad is
a TypeError unless gradients are off (torch.no_grad, torch.inference_mode).
"""
import ctypes

import torch

from .binding import SF_ROPE_AXES, _check, _Rope, load_library

try:
    from . import _operators as _ext
except ImportError as e:
    raise ImportError(f"the binding of the operators does not load ({e}): build it with `python -m paper_2511_22009_amd.build` "
                      "(or __graft_entry__.build())") from e

_TYPES = {torch.bfloat16: 0, torch.float32: 1}
_LAYOUTS = {"adjacent": 0, "halves": 1, "axis_halves": 2}


def _raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


_ext.bind(_check, getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream),
          *(ctypes.cast(getattr(load_library(), "sf_" + n), ctypes.c_void_p).value
            for n in ("quantize_rows", "matmul_i8", "rotate", "qk_norm_rotate")))


def _aside(stream, tensors, call, *args):
    """A call on `stream`: its outputs belong to it, and the inputs' memory is kept for it."""
    first = tensors[0]
    if isinstance(first, torch.Tensor) and first.is_cuda and first.get_device() != stream.device.index:
        raise ValueError(f"stream of {stream.device}, tensors on {first.device}")
    with torch.cuda.stream(stream):
        result = call(*args)
    for t in (*tensors, *(result if isinstance(result, tuple) else (result,))):
        if t is not None:
            t.record_stream(stream)
    return result


# ------------------------------------------------------------------------ 8-bit codes

def quantize_rows(x, out=None, scale=None, stream=None):
    """8-bit codes of the rows of x [rows, cols] (bfloat16 or float32, cols adjacent) and
    the fp32 scale of each row: (codes, scale) with x = codes * scale[:, None] nearly.
    codes: int8 [rows, cols], its rows a multiple of 16 bytes apart as `matmul_i8` reads
    them (of 128 from 1024 columns on: a product of 1023 x 777 x 4321 takes 10.4 us then and
    13.9 with rows 4336 bytes apart, three sets of operands in turn; 10.0 and 11.2 with
    one); `out` and `scale` take the results where they are given."""
    if stream is not None:
        return _aside(stream, (x,), _ext.quantize_rows, x, out, scale)
    return _ext.quantize_rows(x, out, scale)


def matmul_i8(a, a_scale, b, b_scale, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """a [M, K] times b [N, K] transposed, both 8-bit codes with a scale per row, plus bias
    [N] (fp32): [M, N] in `dtype` (bfloat16 or float32), or in `out`, whose columns are
    adjacent and whose type then holds."""
    if dtype not in _TYPES:
        raise TypeError(f"dtype: expected torch.bfloat16 or torch.float32, got {dtype}")
    if stream is not None:
        return _aside(stream, (a, a_scale, b, b_scale, bias), _ext.matmul_i8, a, a_scale, b, b_scale, bias, _TYPES[dtype], out)
    return _ext.matmul_i8(a, a_scale, b, b_scale, bias, _TYPES[dtype], out)


# ------------------------------------------------------------------- rotary positions

class Rotary:
    """How heads turn by positions: dims[a] dims of a head turn by axis a (even; the head's
    other dims stay), with frequencies theta^(-2 i / dims[a]), or, with `spread`, one
    range of frequencies shared out over the axes. layout: where the two dims of a pair
    lie, "adjacent" (2j, 2j + 1), "halves" (j, j + pairs) or "axis_halves" (halves within
    the dims of each axis)."""

    def __init__(self, dims, theta=10000.0, layout="adjacent", spread=False):
        self.dims = tuple(int(d) for d in dims)
        if not 1 <= len(self.dims) <= SF_ROPE_AXES or any(d < 0 or d % 2 for d in self.dims):
            raise ValueError(f"dims: expected 1 to {SF_ROPE_AXES} even numbers, got {self.dims}")
        if layout not in _LAYOUTS:
            raise ValueError(f"layout: expected one of {sorted(_LAYOUTS)}, got {layout!r}")
        self.theta, self.layout, self.spread = float(theta), layout, bool(spread)
        self._struct = _Rope(len(self.dims), (ctypes.c_int * SF_ROPE_AXES)(*self.dims), _LAYOUTS[layout], int(self.spread),
                             self.theta)
        self._address = ctypes.addressof(self._struct)

    def __reduce__(self):
        # copies and pickles are made anew: the address of another's struct would outlive it
        return type(self), (self.dims, self.theta, self.layout, self.spread)


def rotate(x, positions, rotary, inverse=False, out=None, stream=None):
    """x [rows, tokens, heads, dims] (bfloat16 or float32, dims adjacent, other strides
    free) with every head turned by its token's position, or turned back (`inverse`).
    positions: fp32 [tokens, axes], or [rows, tokens, axes]. `out` may be x itself."""
    if not isinstance(rotary, Rotary):
        raise TypeError(f"rotary: expected a Rotary, got {type(rotary).__name__}")
    if stream is not None:
        return _aside(stream, (x, positions), _ext.rotate, x, positions, rotary._address, inverse, out)
    return _ext.rotate(x, positions, rotary._address, inverse, out)


def qk_norm_rotate(q, k, q_gain=None, k_gain=None, positions=None, rotary=None, eps=1e-6, out=None, stream=None):
    """Queries q [rows, tokens, heads, dims] and keys k (the same with their own number of
    heads, or None), every head divided by its root mean square (sqrt(mean + eps)),
    multiplied by its gain (fp32 [dims], None: 1) and, with `rotary`, turned by its token's
    position. Returns (q, k); `out` = (q, k) takes the results and may be the inputs (of each its own)."""
    if rotary is not None and not isinstance(rotary, Rotary):
        raise TypeError(f"rotary: expected a Rotary, got {type(rotary).__name__}")
    address = 0 if rotary is None else rotary._address
    q_out, k_out = (None, None) if out is None else out
    if stream is not None:
        return _aside(stream, (q, k, q_gain, k_gain, positions), _ext.qk_norm_rotate, q, k, q_gain, k_gain, positions, address, eps,
                      q_out, k_out)
    return _ext.qk_norm_rotate(q, k, q_gain, k_gain, positions, address, eps, q_out, k_out)
