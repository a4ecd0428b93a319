"""Operators on torch tensors that need no model: 8-bit row quantisation and products,
rotary positions with several axes, and the norm of queries and keys with the rotation
(the calls without a model in include/streamflow.h, which states their formulas).

As in the rest of the binding, tensors give device memory and streams, and shapes, types
and devices are checked before a call: TypeError for what is no fitting tensor, ValueError
for sizes and strides, SFError for what the library refuses. A call runs on the device of
its tensors, on `stream` or torch's current stream there. Outputs that are not given are
allocated for that stream. With a `stream` other than the current one, ordering it after
the work that fills the inputs is the caller's, as in torch; the inputs' memory is kept
until the stream is done with it. Nothing is differentiated.
"""
import ctypes

import torch

from .binding import SF_ROPE_AXES, _check, _Heads, _Rope, load_library

_TYPES = {torch.bfloat16: 0, torch.float32: 1}
_LAYOUTS = {"adjacent": 0, "halves": 1, "axis_halves": 2}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # no Stream object on the way


def _tensor(t, what, dtypes):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what}: expected {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    return t


def _vector(t, what, n, device):
    _tensor(t, what, (torch.float32,))
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {n} adjacent values, got shape {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, the call is on {device}")
    return t.data_ptr()


class _Call:
    """Device and stream of a call; makes the device current where it is not."""
    __slots__ = ("device", "stream", "raw", "_guard")

    def __init__(self, device, stream):
        self.device, self._guard = device, None
        if stream is not None and stream.device != device:
            raise ValueError(f"stream of {stream.device}, tensors on {device}")
        self.raw = (_raw_stream(device.index) if _raw_stream is not None
                    else torch.cuda.current_stream(device).cuda_stream)
        self.stream = None
        if stream is not None and stream.cuda_stream != self.raw:
            self.stream, self.raw = stream, stream.cuda_stream

    def empty(self, make):
        if self.stream is None:
            return make()
        with torch.cuda.stream(self.stream):
            return make()

    def run(self, name, inputs, *args):
        fn = getattr(load_library(), name)
        if self.device.index == torch.cuda.current_device():
            rc = fn(*args, self.raw)
        else:
            with torch.cuda.device(self.device):
                rc = fn(*args, self.raw)
        _check(rc, name)
        if self.stream is not None:
            for t in inputs:
                if t is not None:
                    t.record_stream(self.stream)


# ------------------------------------------------------------------------ 8-bit codes

def quantize_rows(x, out=None, scale=None, stream=None):
    """8-bit codes of the rows of x [rows, cols] (bfloat16 or float32, cols adjacent) and
    the fp32 scale of each row: (codes, scale) with x = codes * scale[:, None] nearly.
    codes: int8 [rows, cols], its rows a multiple of 16 bytes apart as `matmul_i8` reads
    them; `out` and `scale` take the results where they are given."""
    _tensor(x, "x", _TYPES)
    if x.dim() != 2 or x.shape[1] < 1 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"x: expected rows of adjacent values, got shape {tuple(x.shape)}, strides {x.stride()}")
    rows, cols = x.shape
    pitch = -(-cols // 16) * 16
    call = _Call(x.device, stream)
    if out is None:
        out = call.empty(lambda: torch.empty((rows, pitch), dtype=torch.int8, device=x.device))
        ldc = pitch
        if pitch != cols:
            out = out[:, :cols]
    else:
        _tensor(out, "out", (torch.int8,))
        if out.shape != x.shape or out.device != x.device:
            raise ValueError(f"out: expected {tuple(x.shape)} on {x.device}, got {tuple(out.shape)} on {out.device}")
        ldc = _pitch(out, "out", pitch)
    if scale is None:
        scale = call.empty(lambda: torch.empty(rows, dtype=torch.float32, device=x.device))
        ps = scale.data_ptr()
    else:
        ps = _vector(scale, "scale", rows, x.device)
    call.run("sf_quantize_rows", (x, out, scale), x.data_ptr(), _TYPES[x.dtype], rows, cols, x.stride(0), out.data_ptr(), ldc, ps)
    return out, scale


def _pitch(t, what, need):
    """Row length of codes whose rows start at multiples of 16 bytes."""
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: expected rows of adjacent codes, got strides {t.stride()}")
    ld = t.stride(0) if t.shape[0] > 1 else need
    if ld % 16 or ld < need or t.data_ptr() % 16:
        raise ValueError(f"{what}: rows have to start at multiples of 16 bytes, at least {need} apart (strides {t.stride()}); "
                         "quantize_rows leaves them so")
    return ld


def _codes(t, what):
    _tensor(t, what, (torch.int8,))
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{what}: expected codes [rows, cols], got shape {tuple(t.shape)}")
    rows, cols = t.shape
    need = -(-cols // 16) * 16
    ld = _pitch(t, what, need)
    # rows are read in pieces of 16 bytes: the last one's has to lie in the storage too
    if cols != need and rows and t.storage_offset() + (rows - 1) * ld + need > t.untyped_storage().nbytes():
        raise ValueError(f"{what}: the last row ends its storage inside a piece of 16 bytes")
    return ld


def matmul_i8(a, a_scale, b, b_scale, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """a [M, K] times b [N, K] transposed, both 8-bit codes with a scale per row, plus bias
    [N] (fp32): [M, N] in `dtype` (bfloat16 or float32), or in `out`, whose columns are
    adjacent and whose type then holds."""
    lda, ldb = _codes(a, "a"), _codes(b, "b")
    M, K = a.shape
    N = b.shape[0]
    device = a.device
    if b.shape[1] != K or b.device != device:
        raise ValueError(f"b: expected [N, {K}] on {device}, got {tuple(b.shape)} on {b.device}")
    call = _Call(device, stream)
    if out is None:
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected torch.bfloat16 or torch.float32, got {dtype}")
        out = call.empty(lambda: torch.empty((M, N), dtype=dtype, device=device))
        ldo = N
    else:
        _tensor(out, "out", _TYPES)
        ldo = out.stride(0) if M > 1 else N
        if out.shape != (M, N) or out.device != device or (N > 1 and out.stride(1) != 1) or ldo < N:
            raise ValueError(f"out: expected {(M, N)} with adjacent columns on {device}, got {tuple(out.shape)}, "
                             f"strides {out.stride()} on {out.device}")
    call.run("sf_matmul_i8", (a, a_scale, b, b_scale, bias, out), a.data_ptr(), lda, _vector(a_scale, "a_scale", M, device),
             b.data_ptr(), ldb, _vector(b_scale, "b_scale", N, device),
             None if bias is None else _vector(bias, "bias", N, device), M, N, K, out.data_ptr(), ldo, _TYPES[out.dtype])
    return out


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
        self._ref = ctypes.byref(self._struct)


def _heads(x, what, out, call, like=None):
    _tensor(x, what, _TYPES)
    if x.dim() != 4 or (x.shape[3] > 1 and x.stride(3) != 1):
        raise ValueError(f"{what}: expected [rows, tokens, heads, dims] with adjacent dims, got shape {tuple(x.shape)}, "
                         f"strides {x.stride()}")
    if like is not None and (x.shape[:2] != like.shape[:2] or x.shape[3] != like.shape[3] or x.dtype != like.dtype or
                             x.device != like.device):
        raise ValueError(f"{what}: {tuple(x.shape)} of {x.dtype} on {x.device} does not go with {tuple(like.shape)} of "
                         f"{like.dtype} on {like.device}")
    if out is None:
        out = call.empty(lambda: torch.empty_like(x))
    else:
        _tensor(out, what + " out", (x.dtype,))
        if out.shape != x.shape or out.device != x.device or (x.shape[3] > 1 and out.stride(3) != 1):
            raise ValueError(f"{what} out: expected {tuple(x.shape)} with adjacent dims on {x.device}, got {tuple(out.shape)}, "
                             f"strides {out.stride()} on {out.device}")
    si, so = x.stride(), out.stride()
    return out, _Heads(x.data_ptr(), out.data_ptr(), x.shape[2], si[0], si[1], si[2], so[0], so[1], so[2])


def _positions(pos, rotary, x):
    rows, tokens, axes = x.shape[0], x.shape[1], len(rotary.dims)
    _tensor(pos, "positions", (torch.float32,))
    if pos.dim() == 2:
        pos = pos[None]
    if pos.dim() != 3 or pos.shape[0] not in (1, rows) or pos.shape[1] != tokens or pos.shape[2] != axes or pos.device != x.device:
        raise ValueError(f"positions: expected [tokens, axes] or [rows, tokens, axes] = {(rows, tokens, axes)} on {x.device}, got "
                         f"{tuple(pos.shape)} on {pos.device}")
    if (axes > 1 and pos.stride(2) != 1) or (tokens > 1 and pos.stride(1) != axes):
        raise ValueError(f"positions: expected [tokens, axes] without gaps, got strides {pos.stride()}")
    return pos.data_ptr(), pos.stride(0) if pos.shape[0] > 1 else 0


def rotate(x, positions, rotary, inverse=False, out=None, stream=None):
    """x [rows, tokens, heads, dims] (bfloat16 or float32, dims adjacent, other strides
    free) with every head turned by its token's position, or turned back (`inverse`).
    positions: fp32 [tokens, axes], or [rows, tokens, axes]. `out` may be x itself."""
    call = _Call(x.device, stream) if isinstance(x, torch.Tensor) and x.is_cuda else None
    out, h = _heads(x, "x", out, call)
    pos, pos_row = _positions(positions, rotary, x)
    call.run("sf_rotate", (x, positions, out), ctypes.byref(h), _TYPES[x.dtype], x.shape[0], x.shape[1], x.shape[3], rotary._ref,
             pos, pos_row, int(inverse))
    return out


def qk_norm_rotate(q, k, q_gain=None, k_gain=None, positions=None, rotary=None, eps=1e-6, out=None, stream=None):
    """Queries q [rows, tokens, heads, dims] and keys k (the same with their own number of
    heads, or None), every head divided by its root mean square (sqrt(mean + eps)),
    multiplied by its gain (fp32 [dims], None: 1) and, with `rotary`, turned by its token's
    position. Returns (q, k); `out` = (q, k) takes the results and may be the inputs."""
    call = _Call(q.device, stream) if isinstance(q, torch.Tensor) and q.is_cuda else None
    q_out, k_out = out if out is not None else (None, None)
    q_out, hq = _heads(q, "q", q_out, call)
    k_ref = None
    if k is not None:
        k_out, hk = _heads(k, "k", k_out, call, like=q)
        k_ref = ctypes.byref(hk)
    dims, device = q.shape[3], q.device
    gq = None if q_gain is None else _vector(q_gain, "q_gain", dims, device)
    gk = None if k_gain is None else _vector(k_gain, "k_gain", dims, device)
    pos, pos_row, ref = None, 0, None
    if rotary is not None:
        if positions is None:
            raise ValueError("positions: needed with rotary")
        pos, pos_row = _positions(positions, rotary, q)
        ref = rotary._ref
    call.run("sf_qk_norm_rotate", (q, k, q_gain, k_gain, positions, q_out, k_out), ctypes.byref(hq), k_ref, gq, gk, float(eps),
             _TYPES[q.dtype], q.shape[0], q.shape[1], dims, ref, pos, pos_row)
    return q_out, k_out if k is not None else None
