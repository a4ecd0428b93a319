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

_T = torch.Tensor
_BF16, _FP32, _INT8 = torch.bfloat16, torch.float32, torch.int8
_TYPES = {_BF16: 0, _FP32: 1}
_LAYOUTS = {"adjacent": 0, "halves": 1, "axis_halves": 2}

# A call's checks and allocations take the host about as long as its launch, and the smallest
# calls no longer than that on the GPU, so what a call asks for is asked for once and in the
# cheapest form: dtypes by identity, strides as one tuple, the raw stream without its object.


def _raw_stream(index):
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


def _stream_of(index, stream):
    """The raw stream of a call, and `stream` itself where it is not the current one."""
    raw = _raw_stream(index)
    if stream is None:
        return raw, None
    if stream.device.index != index:
        raise ValueError(f"stream of {stream.device}, tensors on cuda:{index}")
    return stream.cuda_stream, None if stream.cuda_stream == raw else stream


def _empty(side, sizes, strides, dtype, device):
    if side is None:
        return torch.empty_strided(sizes, strides, dtype=dtype, device=device)
    with torch.cuda.stream(side):
        return torch.empty_strided(sizes, strides, dtype=dtype, device=device)


def _run(name, index, side, tensors, *args):
    fn = getattr(load_library(), name)
    if index == torch.cuda.current_device():
        rc = fn(*args)
    else:
        with torch.cuda.device(index):
            rc = fn(*args)
    if rc:
        _check(rc, name)
    if side is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(side)


def _tensor(t, what, dtypes):
    if not isinstance(t, _T) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what}: expected {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")


def _vector(t, what, n, index):
    """Address of n adjacent fp32 values."""
    if not (isinstance(t, _T) and t.is_cuda and t.dtype is _FP32):
        _tensor(t, what, (_FP32,))
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {n} adjacent values, got shape {tuple(t.shape)}")
    if t.get_device() != index:
        raise ValueError(f"{what}: on {t.device}, the call is on cuda:{index}")
    return t.data_ptr()


# ------------------------------------------------------------------------ 8-bit codes

def quantize_rows(x, out=None, scale=None, stream=None):
    """8-bit codes of the rows of x [rows, cols] (bfloat16 or float32, cols adjacent) and
    the fp32 scale of each row: (codes, scale) with x = codes * scale[:, None] nearly.
    codes: int8 [rows, cols], its rows a multiple of 16 bytes apart as `matmul_i8` reads
    them (of 128 from 1024 columns on: products of 4321 columns take 9.4 us then, 11.2 with
    rows 4336 bytes apart); `out` and `scale` take the results where they are given."""
    if not (isinstance(x, _T) and x.is_cuda and x.dtype in _TYPES):
        _tensor(x, "x", _TYPES)
    shape, strides = x.shape, x.stride()
    if len(shape) != 2 or shape[1] < 1 or (shape[1] > 1 and strides[1] != 1):
        raise ValueError(f"x: expected rows of adjacent values, got shape {tuple(shape)}, strides {strides}")
    rows, cols = shape
    pitch = (cols + 15) // 16 * 16
    index = x.get_device()
    raw, side = _stream_of(index, stream)
    if out is None:
        ldc = pitch if cols < 1024 else (cols + 127) // 128 * 128  # whole cache lines
        out = _empty(side, (rows, ldc), (ldc, 1), _INT8, x.device)
        if ldc != cols:
            out = out[:, :cols]
    else:
        _tensor(out, "out", (_INT8,))
        if out.shape != shape or out.get_device() != index:
            raise ValueError(f"out: expected {tuple(shape)} on {x.device}, got {tuple(out.shape)} on {out.device}")
        ldc = _pitch(out, "out", pitch)
    if scale is None:
        scale = _empty(side, (rows,), (1,), _FP32, x.device)
        to = scale.data_ptr()
    else:
        to = _vector(scale, "scale", rows, index)
    _run("sf_quantize_rows", index, side, (x, out, scale), x.data_ptr(), _TYPES[x.dtype], rows, cols, strides[0], out.data_ptr(),
         ldc, to, raw)
    return out, scale


def _pitch(t, what, need):
    """Row length of codes whose rows start at multiples of 16 bytes."""
    shape, strides = t.shape, t.stride()
    if shape[1] > 1 and strides[1] != 1:
        raise ValueError(f"{what}: expected rows of adjacent codes, got strides {strides}")
    ld = strides[0] if shape[0] > 1 else need
    if ld % 16 or ld < need or t.data_ptr() % 16:
        raise ValueError(f"{what}: rows have to start at multiples of 16 bytes, at least {need} apart (strides {strides}); "
                         "quantize_rows leaves them so")
    return ld


def _codes(t, what):
    if not (isinstance(t, _T) and t.is_cuda and t.dtype is _INT8):
        _tensor(t, what, (_INT8,))
    shape = t.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{what}: expected codes [rows, cols], got shape {tuple(shape)}")
    rows, cols = shape
    need = (cols + 15) // 16 * 16
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
    index = a.get_device()
    if b.shape[1] != K or b.get_device() != index:
        raise ValueError(f"b: expected [N, {K}] on {a.device}, got {tuple(b.shape)} on {b.device}")
    raw, side = _stream_of(index, stream)
    sa, sb = _vector(a_scale, "a_scale", M, index), _vector(b_scale, "b_scale", N, index)
    to_bias = None if bias is None else _vector(bias, "bias", N, index)
    if out is None:
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected torch.bfloat16 or torch.float32, got {dtype}")
        out = _empty(side, (M, N), (N, 1), dtype, a.device)
        ldo = N
    else:
        _tensor(out, "out", _TYPES)
        dtype = out.dtype
        ldo = out.stride(0) if M > 1 else N
        if out.shape != (M, N) or out.get_device() != index or (N > 1 and out.stride(1) != 1) or ldo < N:
            raise ValueError(f"out: expected {(M, N)} with adjacent columns on {a.device}, got {tuple(out.shape)}, "
                             f"strides {out.stride()} on {out.device}")
    _run("sf_matmul_i8", index, side, (a, a_scale, b, b_scale, bias, out), a.data_ptr(), lda, sa, b.data_ptr(), ldb, sb, to_bias,
         M, N, K, out.data_ptr(), ldo, _TYPES[dtype], raw)
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


def _check_heads(x, what):
    if not (isinstance(x, _T) and x.is_cuda and x.dtype in _TYPES):
        _tensor(x, what, _TYPES)
    shape = x.shape
    if len(shape) != 4 or (shape[3] > 1 and x.stride(3) != 1):
        raise ValueError(f"{what}: expected [rows, tokens, heads, dims] with adjacent dims, got shape {tuple(shape)}, "
                         f"strides {x.stride()}")
    return shape


def _heads(x, what, out, side):
    """The output for x, and both as the library takes them."""
    if out is None:
        if side is None:
            out = torch.empty_like(x)
        else:
            with torch.cuda.stream(side):
                out = torch.empty_like(x)
        so = out.stride()
        if so[3] != 1:  # an x whose entries overlap (windows): its strides' order is not the output's
            n, t, h, d = x.shape
            so = (t * h * d, h * d, d, 1)
            out = _empty(side, x.shape, so, x.dtype, x.device)
    else:
        _tensor(out, what + " out", (x.dtype,))
        so = out.stride()
        if out.shape != x.shape or out.get_device() != x.get_device() or (x.shape[3] > 1 and so[3] != 1):
            raise ValueError(f"{what} out: expected {tuple(x.shape)} with adjacent dims on {x.device}, got {tuple(out.shape)}, "
                             f"strides {so} on {out.device}")
    si = x.stride()
    return out, _Heads(x.data_ptr(), out.data_ptr(), x.shape[2], si[0], si[1], si[2], so[0], so[1], so[2])


def _positions(pos, rotary, shape, index):
    if not isinstance(rotary, Rotary):
        raise TypeError(f"rotary: expected a Rotary, got {type(rotary).__name__}")
    if not (isinstance(pos, _T) and pos.is_cuda and pos.dtype is _FP32):
        _tensor(pos, "positions", (_FP32,))
    rows, tokens, axes = shape[0], shape[1], len(rotary.dims)
    ps, st = pos.shape, pos.stride()
    if len(ps) == 2:
        ps, st = (1, *ps), (0, *st)
    if len(ps) != 3 or ps[0] not in (1, rows) or ps[1] != tokens or ps[2] != axes or pos.get_device() != index:
        raise ValueError(f"positions: expected [tokens, axes] or [rows, tokens, axes] = {(rows, tokens, axes)} on cuda:{index}, got "
                         f"{tuple(pos.shape)} on {pos.device}")
    if (axes > 1 and st[2] != 1) or (tokens > 1 and st[1] != axes):
        raise ValueError(f"positions: expected [tokens, axes] without gaps, got strides {pos.stride()}")
    return pos.data_ptr(), st[0] if ps[0] > 1 else 0


def rotate(x, positions, rotary, inverse=False, out=None, stream=None):
    """x [rows, tokens, heads, dims] (bfloat16 or float32, dims adjacent, other strides
    free) with every head turned by its token's position, or turned back (`inverse`).
    positions: fp32 [tokens, axes], or [rows, tokens, axes]. `out` may be x itself."""
    shape = _check_heads(x, "x")
    index = x.get_device()
    pos, pos_row = _positions(positions, rotary, shape, index)
    raw, side = _stream_of(index, stream)
    out, h = _heads(x, "x", out, side)
    _run("sf_rotate", index, side, (x, positions, out), ctypes.byref(h), _TYPES[x.dtype], shape[0], shape[1], shape[3], rotary._ref,
         pos, pos_row, 1 if inverse else 0, raw)
    return out


def qk_norm_rotate(q, k, q_gain=None, k_gain=None, positions=None, rotary=None, eps=1e-6, out=None, stream=None):
    """Queries q [rows, tokens, heads, dims] and keys k (the same with their own number of
    heads, or None), every head divided by its root mean square (sqrt(mean + eps)),
    multiplied by its gain (fp32 [dims], None: 1) and, with `rotary`, turned by its token's
    position. Returns (q, k); `out` = (q, k) takes the results and may be the inputs (of each its own)."""
    shape = _check_heads(q, "q")
    rows, tokens, _, dims = shape
    index, dtype = q.get_device(), q.dtype
    if k is not None:
        ks = _check_heads(k, "k")
        if ks[0] != rows or ks[1] != tokens or ks[3] != dims or k.dtype is not dtype or k.get_device() != index:
            raise ValueError(f"k: {tuple(ks)} of {k.dtype} on {k.device} does not go with q: {tuple(shape)} of {dtype} on {q.device}")
    gq = None if q_gain is None else _vector(q_gain, "q_gain", dims, index)
    gk = None if k_gain is None else _vector(k_gain, "k_gain", dims, index)
    if rotary is None:
        pos, pos_row, ref = None, 0, None
    else:
        if positions is None:
            raise ValueError("positions: needed with rotary")
        pos, pos_row = _positions(positions, rotary, shape, index)
        ref = rotary._ref
    raw, side = _stream_of(index, stream)
    q_out, k_out = (None, None) if out is None else out
    q_out, hq = _heads(q, "q", q_out, side)
    if k is None:
        k_out = k_ref = None
    else:
        k_out, hk = _heads(k, "k", k_out, side)
        k_ref = ctypes.byref(hk)
    _run("sf_qk_norm_rotate", index, side, (q, k, q_gain, k_gain, positions, q_out, k_out), ctypes.byref(hq), k_ref, gq, gk, eps,
         _TYPES[dtype], rows, tokens, dims, ref, pos, pos_row, raw)
    return q_out, k_out
