"""Operators without a model at the edges of their ranges: heads whose squares leave fp32's,
gains that are not finite, tensors that are no plain ones, calls that take long.

Tolerances as in test_gpu_operators.py.
"""
import numpy as np
import pytest

from test_gpu_operators import BF16, DTYPES, FP32, HALF, NORM, gen, ids, plain_qk, plain_turn, positions, randn, worst

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402

# sizes of heads for each eps: mean squares (and eps itself) below fp32's normal numbers, among
# them heads of subnormal elements ("tiny"), above its largest, and ordinary ones beside them
FAR = [(0.0, [1.0, 1e-19, 1e-22, 1e-30, 1e-37, "tiny", 1e19, 1e25, 3e37]), (1e-40, [1.0, 1e-19, 1e-22, 1e-30, 1e-37, 0.0, 1e25]),
       (1e-30, [1.0, 1e-30, 1e-15, 1e-10, 0.0, 1e25]), (1e-6, [1.0, 1e-30, 1e-3, 0.0, 1e19, 1e25, 3e37]), (3e38, [1e20, 1e15, 1e25, 0.0])]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("dims,layout,dh", [([32, 32], "halves", 64), ([24, 24], "adjacent", 72), ([18, 18], "halves", 36), ([50, 40], "axis_halves", 98),
                                            ([256], "adjacent", 256), ([2], "adjacent", 2)])
def test_norm_of_heads_whose_squares_leave_the_range(dims, layout, dh, dtype):
    """Scaling by a power of two is exact, so the roundings are those of any other head (NORM); an
    ordinary head has the same bits whatever heads it stands beside."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    g = gen(100 + dh)
    r, T, H = Rotary(dims, layout=layout), 21, 16
    pos = positions(g, 1, T, len(dims))
    gain = 1 + 0.3 * randn(g, dh)
    for eps, sizes in FAR:
        eps = float(np.float32(eps))
        tiny = 2.0 ** -140 if dtype == FP32 else 2.0 ** -130
        size = torch.tensor([tiny if s == "tiny" else s for s in sizes], dtype=torch.float64, device="cuda")
        at = torch.randint(len(sizes), (1, T, H, 1), generator=g, device="cuda")
        plain = randn(g, 1, T, H, dh).double()
        plain = torch.sign(plain) * plain.abs().clamp_min(0.5)       # no head is all zero by rounding
        q = (plain * size[at]).to(dtype)
        for x in (q, q.transpose(1, 2).contiguous().transpose(1, 2)):
            for rotary in (r, None):
                got, _ = qk_norm_rotate(x, None, gain, None, pos, rotary, eps=eps)
                want = plain_qk(x, gain, eps)
                want, pair = (want, want.abs()) if rotary is None else plain_turn(want, pos, dims, layout)
                assert worst(got, want, NORM * pair + HALF[dtype] * want.abs()) <= 1.0
        if 1.0 in sizes:
            ordinary = at[..., 0] == sizes.index(1.0)
            beside = q.clone()
            beside[~ordinary] = 1.0
            got, _ = qk_norm_rotate(q, None, gain, None, pos, r, eps=eps)
            alone, _ = qk_norm_rotate(beside, None, gain, None, pos, r, eps=eps)
            assert torch.equal(got[ordinary], alone[ordinary])


def test_norm_of_far_heads_that_are_not_finite():
    """An infinity divides the finite dims of its head to 0 and itself to NaN, as the formula does;
    a NaN takes its head, and heads of other sizes beside them are as alone."""
    from paper_2511_22009_amd import qk_norm_rotate
    x = randn(gen(101), 1, 9, 4, 64) * 1e-25
    want, _ = qk_norm_rotate(x, None, eps=0.0)
    y = x.clone()
    y[0, 2, 1, 5] = float("inf")
    y[0, 3, 0, 7] = float("nan")
    got, _ = qk_norm_rotate(y, None, eps=0.0)
    assert torch.isnan(got[0, 2, 1, 5]) and torch.isnan(got[0, 3, 0]).all()
    got[0, 2, 1, 5] = 0.0
    assert not got[0, 2, 1].any()
    got[0, 2, 1], got[0, 3, 0] = want[0, 2, 1], want[0, 3, 0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("dims,dh", [([32], 64), ([6, 4], 18)])
def test_gains_of_dims_that_stay_are_their_own(dims, dh, bad, dtype):
    """A gain that is not finite on a dim that no pair turns changes that dim alone."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    for layout in ("adjacent", "halves", "axis_halves"):
        g = gen(102)
        r, pos = Rotary(dims, layout=layout), positions(g, 2, 7, len(dims))
        q, gain = randn(g, 2, 7, 3, dh, dtype=dtype), 1 + 0.2 * randn(g, dh)
        want, _ = qk_norm_rotate(q, None, gain, None, pos, r)
        for d in (sum(dims), dh - 1):
            far = gain.clone()
            far[d] = bad
            got, _ = qk_norm_rotate(q, None, far, None, pos, r)
            assert not torch.isfinite(got[..., d]).any()
            got[..., d] = want[..., d]
            assert torch.equal(got, want)


def calls(x, codes, scale, h, pos, gain):
    """Every operator's call with each of its tensors in turn replaced by f of it."""
    from paper_2511_22009_amd import Rotary, matmul_i8, qk_norm_rotate, quantize_rows, rotate
    r = Rotary([32, 32])
    yield lambda f: quantize_rows(f(x))
    yield lambda f: quantize_rows(x, scale=f(scale))
    yield lambda f: matmul_i8(codes, f(scale), codes, scale)
    yield lambda f: matmul_i8(codes, scale, codes, f(scale))
    yield lambda f: matmul_i8(codes, scale, codes, scale, f(scale))
    yield lambda f: matmul_i8(codes, scale, codes, scale, out=f(torch.empty((4, 4), device="cuda")))
    yield lambda f: rotate(f(h), pos, r)
    yield lambda f: rotate(h, f(pos), r)
    yield lambda f: rotate(h, pos, r, out=f(h.clone()))
    yield lambda f: qk_norm_rotate(f(h), h, gain, gain, pos, r)
    yield lambda f: qk_norm_rotate(h, f(h), gain, gain, pos, r)
    yield lambda f: qk_norm_rotate(h, h, f(gain), gain, pos, r)
    yield lambda f: qk_norm_rotate(h, h, gain, f(gain), pos, r)
    yield lambda f: qk_norm_rotate(h, h, gain, gain, f(pos), r)
    yield lambda f: qk_norm_rotate(h, None, out=(f(h.clone()), None))


def call_inputs():
    from paper_2511_22009_amd import quantize_rows
    g = gen(103)
    x = randn(g, 4, 32)
    return x, *quantize_rows(x), randn(g, 2, 3, 4, 64), positions(g, 1, 3, 2)[0], 1 + 0.2 * randn(g, 64)


def test_tensors_that_require_grad_are_refused_while_gradients_are_recorded():
    """Nothing is differentiated, so a gradient would be lost without a word."""
    for call in calls(*call_inputs()):
        with pytest.raises(TypeError, match="requires grad"):
            call(lambda t: t.detach().clone().requires_grad_())
        call(lambda t: t.detach().clone().requires_grad_().detach())
        with torch.no_grad():
            want = call(lambda t: t)
            got = call(lambda t: t.detach().clone().requires_grad_())
        for a, b in zip(*((v if isinstance(v, tuple) else (v,)) for v in (got, want))):
            assert a is None and b is None or torch.equal(a, b)


def test_tensors_with_a_lazy_negation_are_refused():
    """Their memory holds the values' opposites."""
    for call in calls(*call_inputs()):
        with pytest.raises(TypeError, match="negat"):
            call(torch._neg_view)
        call(lambda t: torch._neg_view(t.clone()).resolve_neg())
    # one that public calls make: the imaginary part of a conjugate
    from paper_2511_22009_amd import quantize_rows
    z = torch.complex(randn(gen(104), 6), randn(gen(105), 6))
    with pytest.raises(TypeError, match="negat"):
        quantize_rows(z.conj().imag[:, None])


WAITS = r"""
#include <time.h>
volatile int flag = 0;
extern "C" int wait_for_flag() {
  struct timespec t = {0, 1000000};
  for (int i = 0; i < 5000 && !flag; ++i) nanosleep(&t, 0);
  return flag ? 0 : -1;
}
"""


def test_other_threads_run_while_a_call_is_under_way(tmp_path):
    """In the place of the library's entry points stands a function that waits (5 s at most) for what
    another Python thread does. Nothing is launched."""
    import ctypes
    import subprocess
    import threading

    from paper_2511_22009_amd import operators
    src, lib = str(tmp_path / "w.cpp"), str(tmp_path / "w.so")
    with open(src, "w") as f:
        f.write(WAITS)
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", src, "-o", lib], check=True)
    w = ctypes.CDLL(lib)
    flag = ctypes.c_int.in_dll(w, "flag")
    inputs = call_inputs()
    address = ctypes.cast(w.wait_for_flag, ctypes.c_void_p).value
    entries = [ctypes.cast(getattr(operators.load_library(), "sf_" + n), ctypes.c_void_p).value
               for n in ("quantize_rows", "matmul_i8", "rotate", "qk_norm_rotate")]
    raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", operators._raw_stream)
    try:
        operators._ext.bind(operators._check, raw_stream, *[address] * 4)
        for call in calls(*inputs):
            flag.value = 0
            setter = threading.Timer(0.02, lambda: setattr(flag, "value", 1))
            setter.start()
            call(lambda t: t)                      # SFError after 5 s if no other thread could run
            setter.join()
    finally:
        operators._ext.bind(operators._check, raw_stream, *entries)
    x = randn(gen(106), 4, 32)
    codes, scale = operators.quantize_rows(x)          # the library's own again
    assert float((codes * scale[:, None] - x).abs().max()) <= float(x.abs().max()) / 250


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", [(700, 3001, 1300), (1500, 6001, 1300), (2500, 5001, 777), (4096, 2304, 768), (4096, 768, 4608), (1100, 4608, 1152), (1500, 4600, 1152)])
def test_products_have_the_same_bits_in_every_tile(M, N, K, dtype):
    """The whole product in a large tile, against as few rows and columns at a time as take the
    smallest (test_operators_edges_cpu.py asserts which)."""
    from paper_2511_22009_amd import matmul_i8
    g = gen(M + N + K)
    a, b = (torch.randint(-127, 128, (n, (K + 15) // 16 * 16), generator=g, device="cuda").to(torch.int8)[:, :K] for n in (M, N))
    sa, sb, bias = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda"), randn(g, N) * 50
    whole = matmul_i8(a, sa, b, sb, bias, dtype=dtype)
    bare = matmul_i8(a, sa, b, sb, dtype=dtype)
    for m0, m1, n0, n1 in ((0, 64, 0, N), (M - 65, M, 0, N), (M // 2 - 7, M // 2, 0, N), (0, M, 0, 64), (0, M, N - 33, N)):
        part = a[m0:m1], sa[m0:m1], b[n0:n1], sb[n0:n1]
        assert torch.equal(whole[m0:m1, n0:n1], matmul_i8(*part, bias[n0:n1], dtype=dtype))
        assert torch.equal(bare[m0:m1, n0:n1], matmul_i8(*part, dtype=dtype))


def test_long_calls_on_two_streams_at_once():
    """Both streams start behind one event that comes after some milliseconds of work, so that every
    call is queued before the first runs, and each takes tens of us: the streams' kernels run side by side."""
    from paper_2511_22009_amd import Rotary, matmul_i8, qk_norm_rotate, quantize_rows, rotate
    r = Rotary([36, 36], layout="halves")

    def chain(x, w, sw, gain, pos, stream=None):
        a, sa = quantize_rows(x, stream=stream)
        qkv = matmul_i8(a, sa, w, sw, stream=stream).view(4, -1, 24, 72)
        q, k = qk_norm_rotate(qkv[:, :, :8], qkv[:, :, 8:16], gain, gain, pos, r, stream=stream)
        return a, sa, qkv, q, k, rotate(qkv[:, :, 16:], pos, r, inverse=True, stream=stream)
    sets, want = [], []
    for seed in (107, 108):
        g = gen(seed)
        w, sw = quantize_rows(randn(g, 3 * 576, 1152, dtype=BF16))
        sets.append((randn(g, 8192 + 64 * (seed - 107), 1152, dtype=BF16), w, sw, 1 + 0.1 * randn(g, 72),
                     positions(g, 4, 2048 + 16 * (seed - 107), 2, 500.0)))
        want.append([t.clone() for t in chain(*sets[-1])])
    streams = [torch.cuda.Stream() for _ in sets]

    def queue():
        return [[chain(*args, stream=s) for args, s in zip(sets, streams)] for _ in range(8)]
    torch.cuda.synchronize()
    queue()                                                       # the outputs' memory, which the next ones take again
    busy = torch.randn((8192, 8192), device="cuda")
    torch.cuda.synchronize()
    for _ in range(6):
        busy = (busy @ busy).clamp(-1, 1)
    held = torch.cuda.Event()
    held.record()
    for s in streams:
        s.wait_event(held)
    got = queue()
    queued = not held.query()
    torch.cuda.synchronize()
    assert queued, "the work in front ended before the calls were queued"
    for both in got:
        for out, alone in zip(both, want):
            assert all(torch.equal(p, q) for p, q in zip(out, alone))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("heads", [5, 33, 200, 700])
def test_norm_in_place_beside_far_heads(heads, dtype):
    """Results over their inputs, where some heads' squares leave fp32's range and others' results do
    (gains of 0 and 1e-30): every head is treated once, as with outputs apart."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    for dh, layout, T in ((64, "halves", 3), (72, "adjacent", 1500), (36, "halves", 40)):
        g = gen(109 + dh)
        if heads * T > 100000:
            T = 100
        r, pos = Rotary([16, 16], layout=layout), positions(g, 1, T, 2)
        size = torch.tensor([1.0, 1e-25, 1e25], device="cuda")[torch.randint(3, (1, T, heads, 1), generator=g, device="cuda")]
        q = (randn(g, 1, T, heads, dh) * size).to(dtype)
        for gain in (torch.zeros(dh, device="cuda"), torch.full((dh,), 1e-30, device="cuda"), 1 + 0.2 * randn(g, dh)):
            for x in (q, q.transpose(1, 2).contiguous().transpose(1, 2)):
                for rotary in (r, None):
                    want, _ = qk_norm_rotate(x, None, gain, None, pos, rotary, eps=0.0)
                    y = x.clone(memory_format=torch.preserve_format)
                    qk_norm_rotate(y, None, gain, None, pos, rotary, eps=0.0, out=(y, None))
                    assert torch.isfinite(want).all() and torch.equal(y, want)
                    both = x.clone(memory_format=torch.preserve_format)
                    k = torch.ones_like(q)
                    qk_norm_rotate(both, k, gain, None, pos, rotary, eps=0.0, out=(both, k))
                    assert torch.equal(both, want)
