"""The operators without a model against plain 64-bit implementations.

Tolerances count roundings: one of fp32 is at most 2^-24 of its result, one of bf16 2^-8.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402

BF16, FP32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}   # half a step of the type, relative
U = 2.0 ** -24
DTYPES = [BF16, FP32]
ids = lambda v: str(v).replace("torch.", "")  # noqa: E731


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=FP32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def worst(got, want, allowed):
    """Largest |got - want| / allowed (0 where both are 0)."""
    d = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all()
    return float((d / allowed.clamp_min(1e-300)).max()) if d.numel() else 0.0


# ------------------------------------------------------------------------ 8-bit codes

def plain_quantize(x):
    """From the definition: the quotient 127 x / a in 64 bits (127 x is exact there, and its
    quotients are halves exactly when the true ones are), ties to even."""
    x = x.double().cpu().numpy()
    a = np.abs(x).max(1)
    q = np.rint(127.0 * x / np.where(a > 0, a, 1.0)[:, None])
    return q.astype(np.int8), a.astype(np.float32) / np.float32(127.0)


def check_quantize(x, **kw):
    from paper_2511_22009_amd import quantize_rows
    codes, scale = quantize_rows(x, **kw)
    q, s = plain_quantize(x)
    assert codes.dtype == torch.int8 and codes.shape == x.shape
    np.testing.assert_array_equal(codes.cpu().numpy(), q)
    np.testing.assert_array_equal(scale.cpu().numpy(), s)
    return codes, scale


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (1, 8), (5, 16), (2, 513), (64, 1152), (7, 770), (33, 4608), (2, 8192), (3, 20011),
                                 (1, 131072), (2500, 40)])
def test_quantize_rows(M, K, dtype):
    g = gen(M * 1000 + K)
    x = randn(g, M, K) * torch.exp(2 * randn(g, M, 1))
    check_quantize(x.to(dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize_rows_of_every_kind(dtype):
    """Zeros, one value, ties (largest magnitudes whose quotients are halves), far scales."""
    g = gen(1)
    x = randn(g, 12, 96)
    x[0] = 0
    x[1] = 0
    x[1, 17] = -3.5
    x[2] = torch.arange(96, device="cuda") * 2.0 + 1.0
    x[2, 5] = 254.0                                     # 127 x / 254 = x / 2: a half at every odd x
    x[3] = x[2] * -0.5
    x[4] *= 1e-30
    x[5] *= 3e37
    x[6] = 1e-38 * torch.sign(x[6])
    x[7] = -x[7].abs()
    x[8] = 2.0 ** -126 * (torch.arange(96, device="cuda") % 3)
    x[9] *= 1e-37
    x[10] = 3.0e38
    x[11, 1:] = 0
    check_quantize(x.to(dtype))


def test_quantize_rows_next_to_halves():
    """fp32 values on both sides of every half, one and a few steps away."""
    a = np.float32(0.7318)
    n = np.arange(-126, 127)
    half = ((n + np.sign(n) * 0.5) * np.float64(a) / 127.0).astype(np.float32)
    rows = [half]
    for k in (1, 2, 5):
        up, down = half.copy(), half.copy()
        for _ in range(k):
            up, down = np.nextafter(up, np.float32(9)), np.nextafter(down, np.float32(-9))
        rows += [up, down]
    x = np.stack(rows)
    x = np.concatenate([x, np.full((len(rows), 1), a)], 1)
    check_quantize(torch.from_numpy(x).cuda())


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_quantize_rows_that_are_not_finite(bad, dtype):
    from paper_2511_22009_amd import quantize_rows
    x = randn(gen(2), 9, 300, dtype=dtype)
    want, scales = plain_quantize(x)
    for row, col in ((0, 0), (4, 299), (7, 150)):
        x[row, col] = bad
    codes, scale = quantize_rows(x)
    for m in range(9):
        if m in (0, 4, 7):
            assert not codes[m].any() and torch.isnan(scale[m])
        else:
            np.testing.assert_array_equal(codes[m].cpu().numpy(), want[m])
            assert float(scale[m]) == scales[m]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize_rows_strides_and_given_outputs(dtype):
    """Columns of wider rows at an odd offset, one row repeated by a stride of 0, and outputs
    inside a larger buffer whose other bytes stay."""
    x = randn(gen(3), 21, 250, dtype=dtype)
    check_quantize(x[:, 1:238])
    check_quantize(x[::2, 3:100])
    check_quantize(x[4:5].expand(6, 250))
    buf = torch.full((25, 272), 77, dtype=torch.int8, device="cuda")
    sc = torch.full((30,), 5.0, device="cuda")
    codes, scale = check_quantize(x[:, 1:238], out=buf[2:23, 16:253], scale=sc[4:25])
    assert codes.data_ptr() == buf[2:23, 16:].data_ptr() and scale.data_ptr() == sc[4:].data_ptr()
    keep = buf.clone()
    keep[2:23, 16:253] = 77
    assert (keep == 77).all() and (sc[:4] == 5).all() and (sc[25:] == 5).all()
    codes, scale = check_quantize(x[:0])
    assert codes.shape == (0, 250) and scale.shape == (0,)


def codes(g, rows, K, pad=None, largest=127):
    """8-bit codes at a row pitch past K, the bytes past K filled with other codes."""
    pitch = (K + 15) // 16 * 16 if pad is None else pad
    q = torch.randint(-largest, largest + 1, (rows, pitch), generator=g, device="cuda").to(torch.int8)
    return q[:, :K]


def check_matmul(a, sa, b, sb, bias, dtype, **kw):
    from paper_2511_22009_amd import matmul_i8
    got = matmul_i8(a, sa, b, sb, bias, dtype=dtype, **kw)
    total = a.double() @ b.double().t()                   # exact: below 2^31
    p = total * sa.double()[:, None] * sb.double()
    want = p if bias is None else p + bias.double()
    # conversion and two products, the sum with the bias, then the rounding to the type
    allowed = 3 * U * p.abs() + U * want.abs() + (HALF[dtype] * want.abs() if dtype != FP32 else 0)
    assert worst(got, want, allowed * 1.01) <= 1.0
    return got


SIZES = [(1, 1, 1), (1, 8, 16), (2, 7, 15), (1, 3456, 1152), (5, 100, 17), (16, 64, 128), (17, 65, 129), (31, 777, 1000), (33, 96, 192),
         (64, 64, 64), (65, 200, 300), (128, 128, 256), (130, 50, 4321), (200, 1152, 768), (257, 129, 513), (1023, 777, 1001),
         (1500, 2304, 768), (4100, 40, 96), (3, 5000, 2000), (8, 1152, 4608), (12, 33, 8192)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_matmul_i8(M, N, K, dtype):
    g = gen(M + 3 * N + 7 * K)
    a, b = codes(g, M, K), codes(g, N, K)
    sa, sb = torch.rand(M, generator=g, device="cuda") + 0.01, torch.rand(N, generator=g, device="cuda") * 0.1
    bias = randn(g, N) * 50 if (M + N + K) % 2 else None
    got = check_matmul(a, sa, b, sb, bias, dtype)
    assert got.dtype == dtype and got.shape == (M, N)
    from paper_2511_22009_amd import matmul_i8
    assert torch.equal(got, matmul_i8(a, sa, b, sb, bias, dtype=dtype))       # the same bits again


# sizes that each tile takes, from 128 x 128 on, ending inside one, K inside a slice: within a
# stage's first fill and long enough for the loop that checks no load
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", [(1999, 2047, 2050), (700, 3001, 260), (700, 3001, 1300), (700, 6001, 129), (700, 6001, 1025), (1500, 6001, 17),
                                   (1500, 6001, 1300), (2500, 5001, 100), (2500, 5001, 777), (2500, 5001, 900)])
def test_matmul_i8_in_large_tiles(M, N, K, dtype):
    g = gen(M + 3 * N + 7 * K)
    a, b = codes(g, M, K), codes(g, N, K)
    sa, sb = torch.rand(M, generator=g, device="cuda") + 0.01, torch.rand(N, generator=g, device="cuda") * 0.1
    out = torch.full((M + 2, N + 8), 3.0, dtype=dtype, device="cuda")
    check_matmul(a, sa, b, sb, randn(g, N) * 50, dtype, out=out[1:-1, 3:N + 3])
    out[1:-1, 3:N + 3] = 3.0
    assert (out == 3.0).all()                                                  # nothing around it is touched


def test_matmul_i8_a_row_does_not_depend_on_the_others():
    """The sums are exact, so a token's outputs are the same bits however many there are."""
    from paper_2511_22009_amd import matmul_i8
    g = gen(9)
    a, b = codes(g, 700, 1000), codes(g, 385, 1000)
    sa, sb, bias = torch.rand(700, device="cuda"), torch.rand(385, device="cuda"), randn(g, 385)
    for dtype in DTYPES:
        whole = matmul_i8(a, sa, b, sb, bias, dtype=dtype)
        for lo, hi in ((0, 1), (5, 20), (100, 165), (300, 700)):
            assert torch.equal(whole[lo:hi], matmul_i8(a[lo:hi], sa[lo:hi], b, sb, bias, dtype=dtype))


@pytest.mark.parametrize("M,N", [(1, 3), (20, 40), (70, 130)])
def test_matmul_i8_longest_sum_of_the_largest_codes(M, N):
    """131071 products of -128 and -128: 2^31 less 2^14, the last sum that 32 bits hold."""
    from paper_2511_22009_amd import matmul_i8
    K = 131071
    a = torch.full((M, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    b = torch.full((N, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    one = torch.ones(max(M, N), device="cuda")
    got = matmul_i8(a, one[:M], b, one[:N], dtype=FP32)
    assert (got.double() == float(np.float32(2 ** 31 - 2 ** 14))).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", [(1, 50, 100), (9, 130, 300), (70, 33, 200), (300, 257, 129)])
def test_matmul_i8_strides_and_given_output(M, N, K, dtype):
    """Operands inside wider rows, an output inside a larger one at an odd place, whose other
    elements stay."""
    g = gen(M * N)
    a, b = codes(g, M, K, pad=512), codes(g, N, K, pad=336)
    sa, sb, bias = torch.rand(M, device="cuda"), torch.rand(N, device="cuda"), randn(g, N)
    buf = torch.full((M + 4, N + 9), 7.0, dtype=dtype, device="cuda")
    check_matmul(a, sa, b, sb, bias, dtype, out=buf[2:M + 2, 3:N + 3])
    buf[2:M + 2, 3:N + 3] = 7.0
    assert (buf == 7.0).all()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_matmul_i8_of_rows_that_are_not_finite(M):
    """A scale of NaN (a row that was not finite) makes that row NaN and no other."""
    from paper_2511_22009_amd import matmul_i8
    g = gen(4)
    a, b = codes(g, M, 200), codes(g, 70, 200)
    sa, sb = torch.rand(M, device="cuda"), torch.rand(70, device="cuda")
    a[0] = 0
    sa[0] = float("nan")
    got = matmul_i8(a, sa, b, sb)
    assert torch.isnan(got[0]).all() and torch.isfinite(got[1:]).all()


def test_matmul_i8_past_32_bits():
    """Operands and outputs whose last rows lie more than 2^31 elements in."""
    from paper_2511_22009_amd import matmul_i8
    g = gen(6)
    M, N, K = 280000, 8200, 64
    a = torch.zeros((M, 8192), dtype=torch.int8, device="cuda")[:, :K]
    a[-300:] = codes(g, 300, K)
    b = codes(g, N, K)
    sa, sb = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    assert M * 8192 > 2 ** 31 and M * N > 2 ** 31
    got = matmul_i8(a, sa, b, sb)
    tail = matmul_i8(a[-300:], sa[-300:], b, sb)
    assert torch.equal(got[-300:], tail) and tail.abs().sum() > 0
    assert not got[:1000].any() and not got[-1300:-300].any()


def test_quantized_product_is_near_the_real_one():
    """quantize_rows and matmul_i8 together. Codes are off by at most half a step of
    a / 127, so the product of row m with row n is off by at most
    sum_k (|x| e_w + |w| e_x + e_x e_w), e = a / 254."""
    from paper_2511_22009_amd import matmul_i8, quantize_rows
    g = gen(5)
    x, w = randn(g, 300, 768, dtype=BF16), randn(g, 500, 768, dtype=BF16) * 0.02
    got = matmul_i8(*quantize_rows(x), *quantize_rows(w), dtype=FP32)
    X, W = x.double(), w.double()
    ex, ew = X.abs().amax(1) / 254, W.abs().amax(1) / 254
    allowed = X.abs().sum(1)[:, None] * ew + W.abs().sum(1) * ex[:, None] + 768 * ex[:, None] * ew
    assert worst(got, X @ W.t(), allowed * 1.0001) <= 1.0


# ------------------------------------------------------------------- rotary positions

def pairs_of(dims, layout):
    P, lo, hi, axis, base = sum(dims) // 2, [], [], [], 0
    for a, d in enumerate(dims):
        for i in range(d // 2):
            j = base // 2 + i
            lo.append({"adjacent": 2 * j, "halves": j, "axis_halves": base + i}[layout])
            hi.append({"adjacent": 2 * j + 1, "halves": j + P, "axis_halves": base + d // 2 + i}[layout])
            axis.append(a)
        base += d
    return lo, hi, axis


def plain_turn(x, pos, dims, layout, theta=10000.0, spread=False, inverse=False):
    """x in fp64; also the size |a| + |b| of every element's pair, which its error goes by."""
    lo, hi, axis = pairs_of(dims, layout)
    P = len(lo)
    freq = [theta ** (-j / P) for j in range(P)] if spread else [theta ** (-2.0 * i / d) for d in dims for i in range(d // 2)]
    out, size = x.clone(), x.abs()
    if not P:
        return out, size
    lo, hi, axis = (torch.tensor(v, device="cuda") for v in (lo, hi, axis))
    u = pos.double().reshape((-1,) + pos.shape[-2:])[..., axis] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    c, s = torch.cos(u)[:, :, None], torch.sin(u)[:, :, None] * (-1 if inverse else 1)
    a, b = x[..., lo], x[..., hi]
    out[..., lo], out[..., hi] = a * c - b * s, a * s + b * c
    size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return out, size


def positions(g, rows, tokens, axes, far=50.0):
    return torch.floor(torch.rand((rows, tokens, axes), generator=g, device="cuda") * far)


# The angle in quarter turns arrives in fp32 within 2^-25 of a turn's eighth, the Taylor sums
# round a few times on values up to 1: cosines and sines within 4 x 2^-24. Two products and a sum.
TURN = 8 * U
PLANS = [([8], "adjacent", 8), ([64], "halves", 64), ([32, 32], "adjacent", 64), ([36, 36], "halves", 72), ([36, 36], "axis_halves", 72),
         ([16, 56, 56], "adjacent", 128), ([16, 56, 56], "axis_halves", 128), ([32, 32, 32, 32], "halves", 128), ([16, 16], "axis_halves", 48),
         ([24], "halves", 48), ([6, 10], "axis_halves", 16), ([2], "adjacent", 2), ([18, 18], "halves", 36), ([50, 48], "adjacent", 98),
         ([256], "halves", 256), ([100, 60], "axis_halves", 250), ([0, 20, 0, 12], "axis_halves", 40), ([0], "adjacent", 32)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("dims,layout,dh", PLANS)
def test_rotate(dims, layout, dh, dtype):
    from paper_2511_22009_amd import Rotary, rotate
    g = gen(sum(dims) + dh)
    for rows, tokens, heads, far in ((1, 1, 1, 3.0), (2, 37, 3, 100.0), (1, 130, 16, 90000.0)):
        x = randn(g, rows, tokens, heads, dh, dtype=dtype)
        pos = positions(g, rows, tokens, len(dims), far)
        for spread in (False, True):
            r = Rotary(dims, layout=layout, spread=spread)
            got = rotate(x, pos, r)
            want, size = plain_turn(x.double(), pos, dims, layout, spread=spread)
            assert got.dtype == dtype
            assert worst(got, want, TURN * size + HALF[dtype] * want.abs() + 1e-30) <= 1.0
            back = rotate(x, pos, r, inverse=True)
            want, size = plain_turn(x.double(), pos, dims, layout, spread=spread, inverse=True)
            assert worst(back, want, TURN * size + HALF[dtype] * want.abs() + 1e-30) <= 1.0


def test_rotate_positions_that_are_fractions_negative_or_far():
    from paper_2511_22009_amd import Rotary, rotate
    x = randn(gen(11), 1, 7, 2, 64)
    at = torch.tensor([0.5, -3.25, -70000.0, 1e6, 16777215.0, 0.0, 1e-3], device="cuda")
    pos = torch.stack([at, at.flip(0)], 1)
    want, size = plain_turn(x.double(), pos[None], [32, 32], "adjacent")
    # a frequency in fp64 is off by about 2^-50 of itself: 1e-8 of an angle of 2^24
    assert worst(rotate(x, pos, Rotary([32, 32])), want, (TURN + 2e-8) * size) <= 1.0


def test_rotate_there_and_back():
    from paper_2511_22009_amd import Rotary, rotate
    g = gen(12)
    x, pos, r = randn(g, 2, 50, 4, 72), positions(g, 1, 50, 2), Rotary([36, 36], layout="halves")
    back = rotate(rotate(x, pos, r), pos, r, inverse=True)
    _, size = plain_turn(x.double(), pos, [36, 36], "halves")
    assert worst(back, x.double(), 4 * TURN * size) <= 1.0     # twice, on pairs up to sqrt 2 times as large


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout,dh", [("adjacent", 64), ("halves", 72), ("axis_halves", 64), ("adjacent", 50)])
def test_rotate_strides_in_place_and_shared_positions(layout, dh, dtype):
    """Head-major tensors, slices of packed rows at an odd offset, one head repeated by a
    stride of 0, results written over the inputs; what lies between stays."""
    from paper_2511_22009_amd import Rotary, rotate
    g = gen(13)
    R, T, H = 3, 21, 5
    dims = [16, 24]
    r = Rotary(dims, layout=layout)
    pos = positions(g, 1, T, 2)[0]
    hm = randn(g, R, H, T, dh, dtype=dtype)
    packed = randn(g, R, T, 3 * H * dh + 7, dtype=dtype)
    for x in (hm.transpose(1, 2), packed[:, :, 3:3 + H * dh].unflatten(2, (H, dh)), hm[:, :1].transpose(1, 2).expand(R, T, 4, dh),
              hm[:1].transpose(1, 2).expand(R, T, H, dh)):
        want, size = plain_turn(x.double(), pos, dims, layout)
        got = rotate(x, pos, r)
        assert worst(got, want, TURN * size + HALF[dtype] * want.abs()) <= 1.0
        same = torch.equal(got, rotate(x, pos.expand(R, T, 2), r)) and torch.equal(got, rotate(x, pos[None].repeat(R, 1, 1), r))
        assert same
    x = packed[:, :, 3:3 + H * dh].unflatten(2, (H, dh))
    want, keep = rotate(x, pos, r), packed.clone()
    assert rotate(x, pos, r, out=x) is x
    assert torch.equal(x, want)
    keep[:, :, 3:3 + H * dh] = packed[:, :, 3:3 + H * dh]
    assert torch.equal(keep, packed)
    out = torch.full((R, H, T + 2, dh + 3), 7.0, dtype=dtype, device="cuda")
    rotate(hm.transpose(1, 2), pos, r, out=out[:, :, 1:T + 1, 2:dh + 2].transpose(1, 2))
    assert torch.equal(out[:, :, 1:T + 1, 2:dh + 2].transpose(1, 2), rotate(hm.transpose(1, 2), pos, r))
    out[:, :, 1:T + 1, 2:dh + 2] = 7.0
    assert (out == 7.0).all()


def test_rotate_keeps_what_is_not_finite_to_its_pair():
    from paper_2511_22009_amd import Rotary, rotate
    x = randn(gen(14), 1, 6, 2, 64)
    pos = positions(gen(15), 1, 6, 1)
    r = Rotary([32])
    want = rotate(x, pos, r)
    y = x.clone()
    y[0, 2, 1, 40] = float("inf")          # a dim that stays
    y[0, 3, 0, 5] = float("nan")           # a pair that turns: dims 4 and 5
    got = rotate(y, pos, r)
    assert got[0, 2, 1, 40] == float("inf") and torch.isnan(got[0, 3, 0, 4:6]).all()
    got[0, 2, 1, 40], got[0, 3, 0, 4:6] = want[0, 2, 1, 40], want[0, 3, 0, 4:6]
    assert torch.equal(got, want)


# ------------------------------------------------------------------ norm of q and k

def plain_qk(x, gain, eps):
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return y if gain is None else y * gain.double()


# the sum of up to 256 squares in a tree (up to 4 in a chain per lane, six exchanges): 12
# roundings, halved by the root; root, division, gain and scaling: 5; with the turn's 8
NORM = 20 * U


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("dims,layout,dh", PLANS)
def test_qk_norm_rotate(dims, layout, dh, dtype):
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    g = gen(1000 + sum(dims) + dh)
    r = Rotary(dims, layout=layout)
    for rows, tokens, Hq, Hk in ((1, 1, 1, 1), (2, 37, 12, 3), (1, 130, 4, 16)):
        q, k = randn(g, rows, tokens, Hq, dh, dtype=dtype) * 5, randn(g, rows, tokens, Hk, dh, dtype=dtype) * 0.1
        gq, gk = 1 + 0.3 * randn(g, dh), 1 + 0.3 * randn(g, dh)
        pos = positions(g, rows, tokens, len(dims), 3000.0)
        got = qk_norm_rotate(q, k, gq, gk, pos, r, eps=1e-5)
        for x, gain, y in ((q, gq, got[0]), (k, gk, got[1])):
            want, size = plain_turn(plain_qk(x, gain, 1e-5), pos, dims, layout)
            assert y.dtype == dtype and worst(y, want, NORM * size + HALF[dtype] * want.abs() + 1e-30) <= 1.0


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("dh", [2, 8, 40, 64, 72, 98, 128, 256])
def test_qk_norm_alone_and_without_gains(dh, dtype):
    from paper_2511_22009_amd import qk_norm_rotate
    g = gen(dh)
    q, k = randn(g, 2, 19, 6, dh, dtype=dtype), randn(g, 2, 19, 2, dh, dtype=dtype)
    gain = 1 + 0.3 * randn(g, dh)
    for gq, gk in ((None, None), (gain, None), (None, gain)):
        got = qk_norm_rotate(q, k, gq, gk)
        for x, w, y in ((q, gq, got[0]), (k, gk, got[1])):
            want = plain_qk(x, w, 1e-6)
            assert worst(y, want, (NORM + HALF[dtype]) * want.abs() + 1e-30) <= 1.0
    alone, none = qk_norm_rotate(q, None, gain)
    assert none is None and torch.equal(alone, qk_norm_rotate(q, k, gain, gain)[0])


def test_qk_norm_rotate_in_packed_rows_in_place():
    """q and k where a projection left them, written over; v and the gaps stay."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    g = gen(21)
    for dh, layout in ((64, "halves"), (72, "adjacent"), (36, "halves")):
        qkv = randn(g, 2, 33, 4 + 2 + 2, dh, dtype=BF16)
        gq, gk, pos = 1 + 0.1 * randn(g, dh), 1 + 0.1 * randn(g, dh), positions(g, 2, 33, 2)
        r = Rotary([16, 16], layout=layout)
        q, k = qkv[:, :, :4], qkv[:, :, 4:6]
        want = qk_norm_rotate(q, k, gq, gk, pos, r)
        v = qkv[:, :, 6:].clone()
        got = qk_norm_rotate(q, k, gq, gk, pos, r, out=(q, k))
        assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, 6:], v)


def test_qk_norm_of_zero_and_not_finite_heads():
    """A head of zeros stays zero (eps), also with eps 0 it is NaN as 0 / 0 is; NaN stays in
    its head."""
    from paper_2511_22009_amd import qk_norm_rotate
    q = randn(gen(22), 1, 5, 3, 64, dtype=BF16)
    q[0, 1, 2] = 0
    q[0, 3, 0, 7] = float("nan")
    got, _ = qk_norm_rotate(q, None)
    assert not got[0, 1, 2].any() and torch.isnan(got[0, 3, 0]).all()
    rest = torch.ones(5, 3, dtype=torch.bool, device="cuda")
    rest[3, 0] = False
    assert torch.isfinite(got[0][rest]).all()
    assert torch.isnan(qk_norm_rotate(q, None, eps=0.0)[0][0, 1, 2]).all()


def test_rope_past_32_bits():
    """Heads more than 2^31 elements into their tensor."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate
    g = gen(23)
    T, H, dh = 70000, 128, 256
    q = torch.zeros((1, T, H, dh), dtype=BF16, device="cuda")
    assert q.numel() > 2 ** 31
    q[:, -40:] = randn(g, 1, 40, H, dh, dtype=BF16)
    pos = positions(g, 1, T, 1, 1000.0)
    r = Rotary([128], layout="halves")
    got, _ = qk_norm_rotate(q, None, None, None, pos, r)
    tail, _ = qk_norm_rotate(q[:, -40:], None, None, None, pos[:, -40:].contiguous(), r)
    assert torch.equal(got[:, -40:], tail) and not got[:, :1000].any() and not got[:, -1040:-40].any()


def test_empty_tensors():
    from paper_2511_22009_amd import Rotary, matmul_i8, qk_norm_rotate, rotate
    r = Rotary([8])
    z = torch.zeros
    for shape in ((0, 4, 2, 8), (2, 0, 2, 8), (2, 4, 0, 8)):
        x = z(shape, device="cuda")
        pos = z(shape[1], 1, device="cuda")
        assert rotate(x, pos, r).shape == shape and qk_norm_rotate(x, x, None, None, pos, r)[1].shape == shape
    e = z((0, 32), dtype=torch.int8, device="cuda")
    b = z((5, 32), dtype=torch.int8, device="cuda")
    assert matmul_i8(e, z(0, device="cuda"), b, z(5, device="cuda")).shape == (0, 5)
    assert matmul_i8(b, z(5, device="cuda"), e, z(0, device="cuda")).shape == (5, 0)


# ------------------------------------------------------------------ how they are called

def chain(x, w, sw, gq, gk, pos, r, H, stream=None):
    from paper_2511_22009_amd import matmul_i8, qk_norm_rotate, quantize_rows
    a, sa = quantize_rows(x, stream=stream)
    qkv = matmul_i8(a, sa, w, sw, stream=stream).view(1, x.shape[0], 3 * H, -1)
    return qk_norm_rotate(qkv[:, :, :H], qkv[:, :, H:2 * H], gq, gk, pos, r, stream=stream)


def chain_inputs(seed=31):
    from paper_2511_22009_amd import Rotary, quantize_rows
    g = gen(seed)
    H, dh, K, T = 4, 64, 200, 77
    w, sw = quantize_rows(randn(g, 3 * H * dh, K, dtype=BF16))
    return [randn(g, T, K, dtype=BF16), w, sw, 1 + 0.1 * randn(g, dh), 1 + 0.1 * randn(g, dh), positions(g, 1, T, 2),
            Rotary([32, 32], layout="halves"), H]


def test_operators_on_another_stream_and_in_a_graph():
    """The chain of a projection, captured once and replayed with other inputs, with eager
    calls in between, and on a stream given by argument: the same bits as eager calls."""
    args = chain_inputs()
    want = [t.clone() for t in chain(*args)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = chain(*args, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        chain(*args)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            out = chain(*args)
    for seed in (32, 33, 34):
        x = chain_inputs(seed)[0]
        args[0].copy_(x)
        eager = [t.clone() for t in chain(*args)]
        torch.cuda.synchronize()
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_operators_on_two_streams_at_once():
    """Calls under way on two streams share nothing: the bits of calls alone."""
    both = [chain_inputs(seed) for seed in (36, 37)]
    want = [[t.clone() for t in chain(*args)] for args in both]
    streams = [torch.cuda.Stream() for _ in both]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append(chain(*both[i], stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))


def test_operators_one_after_the_other():
    """Tokens to codes, their product with weights, norm and rotation of its queries and keys,
    against the same in 64 bits from the codes. The product is rounded to bf16 before the norm
    (with its 3 fp32 roundings within d = 1.001 2^-8, so a normalised element is off by less than
    2 d / (1 - d) of itself), the result once more: 2.04 2^-8 of the pair and 1.02 2^-8 of the value."""
    from paper_2511_22009_amd import quantize_rows
    for seed in (31, 35):
        x, w, sw, gq, gk, pos, r, H = args = chain_inputs(seed)
        a, sa = quantize_rows(x)
        v = (a.double() @ w.double().t()) * sa.double()[:, None] * sw.double()
        v = v.view(1, x.shape[0], 3 * H, -1)
        for got, gain, part in zip(chain(*args), (gq, gk), (v[:, :, :H], v[:, :, H:2 * H])):
            want, size = plain_turn(plain_qk(part, gain, 1e-6), pos, r.dims, r.layout)
            assert worst(got, want, 2.04 * 2.0 ** -8 * size + 1.02 * 2.0 ** -8 * want.abs()) <= 1.0


@pytest.mark.parametrize("layout,dims", [("adjacent", [8]), ("halves", [4, 4])])
def test_rope_of_overlapping_windows(layout, dims):
    """Inputs whose entries overlap (windows, expanded heads): the outputs have places of their own."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate, rotate
    g = gen(51)
    r, base, pos = Rotary(dims, layout=layout), randn(g, 400), positions(g, 2, 5, len(dims))
    for strides in ((50, 9, 1, 1), (0, 3, 1, 1), (0, 1, 1, 1), (40, 8, 0, 1), (0, 0, 8, 1), (40, 8, 2, 1)):
        x = base.as_strided((2, 5, 4, 8), strides)
        apart = x.clone(memory_format=torch.contiguous_format)
        assert torch.equal(rotate(x, pos, r), rotate(apart, pos, r))
        for got, want in zip(qk_norm_rotate(x, x, None, None, pos, r), qk_norm_rotate(apart, apart, None, None, pos, r)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout", ["adjacent", "halves"])
@pytest.mark.parametrize("dh", [24, 64, 72, 128])
def test_rope_outputs_apart_next_to_each_other_and_off_alignment(dh, layout, dtype):
    """Heads whose tokens follow each other, heads next to each other, at addresses of every kind:
    the same bits, and nothing around the outputs is touched."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate, rotate
    g = gen(55 + dh)
    R, T, H = 2, 45, 5
    r, pos = Rotary([dh // 4 // 2 * 2, dh // 2], layout=layout), positions(g, R, T, 2, 500.0)
    x, gain = randn(g, R, T, H, dh, dtype=dtype), 1 + 0.2 * randn(g, dh)
    want, (normed, _) = rotate(x, pos, r), qk_norm_rotate(x, None, gain, None, pos, r)
    for strides in ((H * T * dh, dh, T * dh), (T * H * dh, H * dh, dh), (T * (H * dh + 3), H * dh + 3, dh)):
        for off in (0, 1, 32):
            room = torch.full((R * T * (H * dh + 3) + 100,), 7.0, dtype=dtype, device="cuda")
            out = room.as_strided((R, T, H, dh), (*strides, 1), off)
            assert torch.equal(rotate(x, pos, r, out=out), want)
            out.fill_(7.0)
            assert (room == 7.0).all()
            out.copy_(x)
            qk_norm_rotate(out, None, gain, None, pos, r, out=(out, None))
            assert torch.equal(out, normed)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("dh", [8, 24, 40, 72])
def test_rope_heads_next_to_each_other_and_apart_are_the_same_bits(dh, dtype):
    """Whichever way a wavefront takes them, with heads and tokens that do not fill the last one."""
    from paper_2511_22009_amd import Rotary, qk_norm_rotate, rotate
    g = gen(56 + dh)
    for R, T, Hq, Hk, layout in ((1, 1, 4, 4, "halves"), (3, 45, 12, 4, "adjacent"), (1, 7, 20, 28, "halves"), (2, 300, 16, 16, "axis_halves")):
        r, pos = Rotary([dh // 8 * 4, dh // 8 * 4], layout=layout), positions(g, R, T, 2, 500.0)
        q, k, gain = randn(g, R, T, Hq, dh, dtype=dtype), randn(g, R, T, Hk, dh, dtype=dtype), 1 + 0.2 * randn(g, dh)
        apart = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k)]
        assert torch.equal(rotate(q, pos, r), rotate(apart[0], pos, r))
        for got, want in zip(qk_norm_rotate(q, k, gain, None, pos, r), qk_norm_rotate(*apart, gain, None, pos, r)):
            assert torch.equal(got, want)
        for got, want in zip(qk_norm_rotate(q, k, gain, gain), qk_norm_rotate(*apart, gain, gain)):
            assert torch.equal(got, want)


# a launch takes 2^23 rows, so these are several
LONG = 2 ** 23


def test_more_rows_to_codes_than_a_launch_takes():
    from paper_2511_22009_amd import quantize_rows
    x = randn(gen(52), LONG + 5, 16, dtype=BF16)
    codes, scale = quantize_rows(x)
    for part in (slice(0, 1000), slice(LONG - 1000, LONG), slice(LONG, LONG + 5)):
        q, s = plain_quantize(x[part])
        np.testing.assert_array_equal(codes[part].cpu().numpy(), q)
        np.testing.assert_array_equal(scale[part].cpu().numpy(), s)


@pytest.mark.parametrize("M,N", [(LONG + 3, 2), (2, LONG + 9), (1, 2 * LONG + 1)])
def test_larger_products_than_a_launch_takes(M, N):
    """Codes of few values: every result is a small whole number, exact in fp32."""
    from paper_2511_22009_amd import matmul_i8
    g = gen(53)
    a, b = (torch.randint(-9, 10, (n, 16), generator=g, device="cuda", dtype=torch.int8) for n in (M, N))
    sa, sb = (torch.randint(1, 5, (n,), generator=g, device="cuda").float() for n in (M, N))
    bias = torch.randint(-50, 50, (N,), generator=g, device="cuda").float()
    got = matmul_i8(a, sa, b, sb, bias, dtype=FP32)
    want = torch.zeros(M, N, dtype=FP32, device="cuda")
    for k in range(16):
        want += a[:, k, None].float() * b[None, :, k].float()
    assert torch.equal(got, want * sa[:, None] * sb + bias)


@pytest.mark.parametrize("rows,tokens", [(2, LONG + 3), (LONG // 4 + 1, 5)])
def test_more_tokens_turned_than_a_launch_takes(rows, tokens):
    from paper_2511_22009_amd import Rotary, qk_norm_rotate, rotate
    g = gen(54)
    r = Rotary([4])
    x, pos = randn(g, rows, tokens, 1, 4, dtype=BF16), positions(g, rows, tokens, 1)
    turned, (normed, _) = rotate(x, pos, r), qk_norm_rotate(x, None, None, None, pos, r)
    for i in {0, rows // 2, rows - 2, rows - 1}:
        for part in (slice(0, 70), slice(max(0, tokens - 70), tokens)):
            y, p = x[i:i + 1, part].contiguous(), pos[i:i + 1, part].contiguous()
            assert torch.equal(turned[i:i + 1, part], rotate(y, p, r))
            assert torch.equal(normed[i:i + 1, part], qk_norm_rotate(y, None, None, None, p, r)[0])
    shared = rotate(x, pos[0], r)
    assert torch.equal(shared[-1, -70:], rotate(x[-1:, -70:], pos[0, -70:], r)[0])


def test_python_refusals():
    from paper_2511_22009_amd import Rotary, SFError, matmul_i8, qk_norm_rotate, quantize_rows, rotate
    g = gen(41)
    x = randn(g, 4, 32)
    with pytest.raises(TypeError):
        quantize_rows(x.half())
    for bad in (x.t(), x[:, :0], x[0]):
        with pytest.raises(ValueError):
            quantize_rows(bad)
    with pytest.raises(ValueError):
        quantize_rows(x, out=torch.empty((4, 40), dtype=torch.int8, device="cuda")[:, :32])
    with pytest.raises(ValueError):
        quantize_rows(x, scale=torch.empty(3, device="cuda"))
    a, sa = quantize_rows(x)
    b, sb = quantize_rows(randn(g, 6, 32))
    with pytest.raises(TypeError):
        matmul_i8(a.float(), sa, b, sb)
    with pytest.raises(TypeError):
        matmul_i8(a, sa, b, sb, dtype=torch.float16)
    with pytest.raises(TypeError):
        matmul_i8(a, sa.double(), b, sb)
    for args in ((a, sb, b, sb), (a, sa, b, sa), (a, sa, b[:, :16], sb), (a[:, 1:17], sa, b[:, :16], sb), (a, sa, b, sb, sa)):
        with pytest.raises(ValueError):
            matmul_i8(*args)
    odd = torch.zeros((5, 20), dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError):
        matmul_i8(odd, torch.ones(5, device="cuda"), odd, torch.ones(5, device="cuda"))   # rows 20 bytes apart
    with pytest.raises(ValueError):
        matmul_i8(odd[:1], torch.ones(1, device="cuda"), torch.zeros((1, 32), dtype=torch.int8, device="cuda")[:, :20],
                  torch.ones(1, device="cuda"), out=torch.empty((2, 1), device="cuda"))
    h = randn(g, 2, 3, 4, 64)
    pos = torch.zeros((3, 2), device="cuda")
    r = Rotary([32, 32])
    with pytest.raises(TypeError):
        rotate(h.half(), pos, r)
    with pytest.raises(TypeError):
        rotate(h, pos.double(), r)
    with pytest.raises(TypeError):
        rotate(h, pos, None)
    for bad in (pos[:, :1], pos[:2], pos[None].expand(3, 3, 2), pos.t().contiguous().t()):
        with pytest.raises(ValueError):
            rotate(h, bad, r)
    with pytest.raises(ValueError):
        rotate(h.transpose(2, 3), pos, r)
    with pytest.raises(ValueError):
        rotate(h, pos, r, out=h[:, :, :2])
    with pytest.raises(SFError):
        rotate(h, pos, r, out=h[:, :, :1].expand(2, 3, 4, 64))
    with pytest.raises(SFError):
        rotate(h[..., :32], pos, r)                     # the plan's dims pass the head's
    with pytest.raises(SFError):
        rotate(h[..., :33], torch.zeros((3, 1), device="cuda"), Rotary([8]))
    with pytest.raises(ValueError):
        qk_norm_rotate(h, h[:, :2], None, None, pos, r)
    with pytest.raises(ValueError):
        qk_norm_rotate(h, h.bfloat16(), None, None, pos, r)
    with pytest.raises(ValueError):
        qk_norm_rotate(h, h, torch.ones(32, device="cuda"), None, pos, r)
    with pytest.raises(ValueError):
        qk_norm_rotate(h, h, None, None, None, r)
    with pytest.raises(SFError):
        qk_norm_rotate(h, h, eps=-1.0)


def test_a_stream_of_another_device_is_refused():
    from types import SimpleNamespace

    from paper_2511_22009_amd import quantize_rows
    other = SimpleNamespace(cuda_stream=torch.cuda.current_stream().cuda_stream, device=torch.device("cuda", 1))
    with pytest.raises(ValueError):
        quantize_rows(torch.ones((2, 16), device="cuda"), stream=other)
