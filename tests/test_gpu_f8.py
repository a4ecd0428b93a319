"""The operators in 8-bit floating point and the norms around a block against plain 64-bit forms.

Tolerances count roundings (f8_util): one of fp32 is at most 2^-24 of its result, one of
bf16 2^-8, one of e4m3 2^-4.
"""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
import f8_util as P  # noqa: E402
from f8_util import BF16, F8, FP32, gen, randn  # noqa: E402

DTYPES = [BF16, FP32]
ids = lambda v: str(v).replace("torch.", "")  # noqa: E731


# ------------------------------------------------------------------------------- to codes

def check_quantize(x, block_rows, **kw):
    from paper_2511_22009_amd import quantize_f8
    q, s = quantize_f8(x, block_rows, **kw)
    want, scale = P.plain_quantize(x, block_rows)
    assert q.dtype == F8 and q.shape == x.shape and s.shape == scale.shape
    assert torch.equal(s, scale)
    assert torch.equal(q.double(), want)
    return q, s


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (1, 8), (16, 128), (17, 129), (2, 513), (64, 1152), (130, 770), (257, 255),
                                 (128, 128), (129, 4608), (3, 20011), (1, 131072), (2500, 40)])
def test_quantize(M, K, dtype, block_rows):
    g = gen(M * 1000 + K)
    check_quantize((randn(g, M, K) * torch.exp(2 * randn(g, M, 1))).to(dtype), block_rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_quantize_of_every_kind(dtype):
    """Zeros, one value, ties, far scales, values below the normal codes."""
    x = randn(gen(1), 14, 256)
    x[0] = 0
    x[1] = 0
    x[1, 17] = -3.5
    n = torch.arange(256, device="cuda")
    x[2] = (n % 128 - 64) * 0.125 + 0.0625              # quotients that are ties: the scale is 1
    x[2, 5], x[2, 200] = 448.0, -448.0
    x[3] = (n % 128 - 64) * 2.0 ** -10                  # ties of the smallest codes
    x[3, 5], x[3, 200] = 448.0, 448.0
    x[4] *= 1e-30
    x[5] *= 7e37
    x[6] = 1e-38 * torch.sign(x[6])
    x[7] = -x[7].abs()
    x[8] = 2.0 ** -126 * (n % 3)
    x[9] *= 1e-37
    x[10] = 3.0e38
    x[11, 1:] = 0
    x[12] = 2.0 ** -133 * (n % 5 - 2)                   # scales below fp32's normal numbers
    x[13, :128] = 2.0 ** -149                           # and one that rounds to 0
    check_quantize(x.to(dtype), 1)


def test_quantize_next_to_ties():
    """fp32 values on both sides of every tie, one and a few steps away, at a scale that is no power of two."""
    top = torch.tensor(0.7318)
    scale = (top / 448).double()
    e4m3 = torch.arange(0, 127, dtype=torch.uint8).view(F8).double()
    tie = ((e4m3[1:] + e4m3[:-1]) / 2 * scale).float()
    rows = [tie]
    for k in (1, 2, 5):
        up, down = tie.clone(), tie.clone()
        for _ in range(k):
            up, down = torch.nextafter(up, torch.tensor(9.0)), torch.nextafter(down, torch.tensor(-9.0))
        rows += [up, down]
    x = torch.stack(rows + [-r for r in rows])
    check_quantize(torch.cat([x, top.expand(len(x), 1)], 1).cuda(), 1)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_quantize_blocks_that_are_not_finite(bad, dtype):
    from paper_2511_22009_amd import quantize_f8
    x = randn(gen(2), 140, 300, dtype=dtype)
    for block_rows in (1, 128):
        want, scales = P.plain_quantize(x, block_rows)
        y = x.clone()
        y[0, 0] = y[135, 299] = bad
        q, s = quantize_f8(y, block_rows)
        m0 = slice(0, block_rows)
        m1 = slice(135, 136) if block_rows == 1 else slice(128, 140)
        assert torch.isnan(q[m0, :128].float()).all() and torch.isnan(q[m1, 256:].float()).all()
        assert torch.isnan(s[0, 0]) and torch.isnan(s[135 // block_rows, 2])
        q, s = q.double(), s.clone()
        for m, c, b in ((m0, slice(0, 128), 0), (m1, slice(256, 300), 2)):
            q[m, c], s[m.start // block_rows, b] = want[m, c], scales[m.start // block_rows, b]
        assert torch.equal(q, want) and torch.equal(s, scales)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_strides_and_given_outputs(block_rows):
    big = randn(gen(3), 200, 999)
    x = big[5:135, 3:400]
    rb, kb = (130, 4) if block_rows == 1 else (2, 4)
    room = torch.full((130, 416), 7.0, device="cuda").to(F8)
    scale = torch.full((rb, 2 * kb + 1), 9.0, device="cuda")
    q, s = check_quantize(x, block_rows, out=room[:, :397], scale=scale[:, 1::2])
    assert q.data_ptr() == room.data_ptr() and s.data_ptr() == scale[:, 1::2].data_ptr()
    assert (room[:, 397:].float() == 7.0).all() and (scale[:, ::2] == 9.0).all()
    check_quantize(x[:1].expand(64, -1), block_rows)  # a stride of 0


# ------------------------------------------------------------------------------- products

def check_matmul(M, N, K, dtype, bias=True, narrow=False, pitch=None):
    from paper_2511_22009_amd import matmul_f8
    g = gen(31 * M + 7 * N + K)
    a, sa = P.codes(g, M, K, pitch=pitch)
    b, sb = P.codes(g, N, K, 128, pitch=pitch)
    if narrow:
        a, b = P.narrow(a), P.narrow(b)
    c = randn(g, N) if bias else None
    out = matmul_f8(a, sa, b, sb, c, dtype=dtype)
    want, err = P.product(a, sa, b, sb, exact=narrow or dtype == FP32)
    if bias:
        want = want + c.double()
        err = err + (want.abs() + err) * P.U
    assert out.dtype == dtype
    P.check(out, want, err, dtype)
    assert torch.equal(out, matmul_f8(a, sa, b, sb, c, dtype=dtype))  # the same bits


SIZES = [(1, 1, 1), (1, 3456, 1152), (2, 17, 15), (16, 16, 16), (17, 100, 127), (33, 48, 128), (64, 129, 129), (5, 300, 4321),
         (65, 64, 128), (65, 65, 17), (100, 1001, 300), (517, 1001, 777), (128, 128, 130), (300, 260, 8333), (129, 770, 1),
         (2048, 1100, 256), (1000, 4100, 127), (4096, 2304, 768), (2500, 4000, 1153), (32, 4096, 4100),
         (2100, 2000, 520), (4699, 786, 1300), (1412, 5554, 520), (1610, 606, 520), (600, 5500, 260),
         (500, 2000, 70), (600, 1536, 1300), (257, 1700, 4300), (20, 500, 4100), (9, 333, 4096), (16, 1500, 4200), (25, 4500, 260)]


@pytest.mark.parametrize("narrow", [False, True], ids=["wide", "narrow"])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_matmul(M, N, K, dtype, narrow):
    check_matmul(M, N, K, dtype, bias=(M + N) % 3 != 0, narrow=narrow)


@pytest.mark.parametrize("M", [16, 128, 1024])
def test_matmul_as_a_whole(M):
    """On a bell's codes, what the matrix cores cut off stays far below what rounding to bf16 costs: against the
    result rounded once, few values differ, each by one step."""
    from paper_2511_22009_amd import matmul_f8
    g = gen(M)
    a, sa = P.codes(g, M, 1152)
    b, sb = P.codes(g, 2176, 1152, 128)
    want, _ = P.product(a, sa, b, sb, exact=True)
    got = matmul_f8(a, sa, b, sb).double()
    # a value is off by half a step: 2^-9 of it on average over a binade, and 1/sqrt(3) of that; 2^-8 holds for every one
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -8
    assert float((matmul_f8(a, sa, b, sb, dtype=FP32).double() - want).norm() / want.norm()) <= 11 * P.U * 2 ** 0.5 * 2


@pytest.mark.parametrize("M", [3, 70, 700])
def test_matmul_rows_far_apart(M):
    check_matmul(M, 333, 200, FP32, pitch=4096)


def test_matmul_that_is_a_selection():
    """Codes of one, at places of their own, pick the other operand's values: exact in fp32."""
    from paper_2511_22009_amd import matmul_f8
    for M, N, K in ((7, 40, 300), (130, 300, 300), (1100, 4200, 384)):
        g = gen(K)
        a, sa = P.codes(g, M, K)
        at = torch.randint(0, K, (N,), generator=g, device="cuda")
        b = torch.zeros((N, -(-K // 16) * 16), device="cuda")
        b[torch.arange(N, device="cuda"), at] = 1.0
        b = b.to(F8)[:, :K]
        sb = torch.ones((-(-N // 128), P.blocks(K)), device="cuda")
        out = matmul_f8(a, sa, b, sb, dtype=FP32)
        assert torch.equal(out, (a.float() * P.spread(sa, M, K))[:, at])


@pytest.mark.parametrize("M", [2, 90, 1024])
def test_matmul_scales_of_every_stride(M):
    from paper_2511_22009_amd import matmul_f8
    g = gen(5)
    a, sa = P.codes(g, M, 700)
    b, sb = P.codes(g, 2100, 700, 128)
    want = matmul_f8(a, sa, b, sb, dtype=FP32)
    wide = torch.full((M, 40), float("nan"), device="cuda")
    wide[:, 3::6] = 0
    wide[:, 3:39:6] = sa
    assert torch.equal(matmul_f8(a, wide[:, 3:39:6], b, sb.contiguous(), dtype=FP32), want)
    one = sa[:1].expand(M, -1)
    assert torch.equal(matmul_f8(a, one, b, sb, dtype=FP32), matmul_f8(a, one.contiguous(), b, sb, dtype=FP32))
    out = torch.full((M, 2200), 5.0, device="cuda", dtype=BF16)
    got = matmul_f8(a, sa, b, sb, out=out[:, 7:2107])
    assert got.data_ptr() == out[:, 7:2107].data_ptr() and torch.equal(got, matmul_f8(a, sa, b, sb))
    assert (out[:, :7] == 5).all() and (out[:, 2107:] == 5).all()


@pytest.mark.parametrize("M", [4, 80, 1024])
def test_matmul_of_codes_that_are_nan(M):
    """A NaN reaches its row, and as a weight its column, and nothing else; so does a NaN scale."""
    from paper_2511_22009_amd import matmul_f8
    g = gen(6)
    a, sa = P.codes(g, M, 260)
    b, sb = P.codes(g, 2100, 260, 128)
    want = matmul_f8(a, sa, b, sb, dtype=FP32)
    a.view(torch.uint8)[1, 259] = 0x7f
    b.view(torch.uint8)[2099, 0] = 0xff
    sa[3, 1] = float("nan")
    sb[1, 2] = float("nan")
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[1] = bad[3] = True
    bad[:, 2099] = bad[:, 128:256] = True
    out = matmul_f8(a, sa, b, sb, dtype=FP32)
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], want[~bad])


# ------------------------------------------------------------------------------- gated projections

def check_gated(M, N, K, dtype, name, bias, narrow=False):
    from paper_2511_22009_amd import gated_matmul_f8
    g = gen(31 * M + 7 * N + K)
    a, sa = P.codes(g, M, K)
    gate, sg = P.codes(g, N, K, 128, size=0.03 / K ** 0.5)
    up, su = P.codes(g, N, K, 128, size=0.03 / K ** 0.5, pitch=-(-K // 128) * 128 + 32)
    if narrow:
        a, gate, up = (P.narrow(q) for q in (a, gate, up))
        sa = sa * 64.0
    bg, bu = (randn(g, N), randn(g, N)) if bias else (None, None)
    call = lambda: gated_matmul_f8(a, sa, gate, sg, up, su, bg, bu, activation=name, dtype=dtype)  # noqa: E731
    out = call()
    want, err = P.gated(a, sa, gate, sg, up, su, bg, bu, name, exact=narrow or dtype != BF16)
    if dtype == F8:
        assert out[0].dtype == F8 and out[0].shape == (M, N) and out[1].shape == (M, P.blocks(N))
        P.check_codes(*out, want, err)
        again = call()
        assert torch.equal(out[0].view(torch.uint8), again[0].view(torch.uint8)) and torch.equal(out[1], again[1])
    else:
        P.check(out, want, err, dtype)
        assert torch.equal(out, call())


@pytest.mark.parametrize("dtype", [BF16, FP32, F8], ids=ids)
@pytest.mark.parametrize("name", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 2048, 768), (16, 17, 33), (20, 130, 129), (64, 300, 128), (65, 33, 300), (200, 129, 144),
                                   (300, 700, 1000), (513, 64, 8320), (1025, 2100, 260), (2304, 2176, 768), (32, 1000, 1152), (800, 600, 140),
                                   (4699, 393, 1300), (646, 2750, 260), (1610, 303, 520), (2048, 550, 256), (500, 1000, 70),
                                   (590, 700, 2309), (8, 300, 4222), (30, 260, 4100)])
def test_gated(M, N, K, name, dtype):
    check_gated(M, N, K, dtype, name, bias=(M + N) % 2 == 1)
    check_gated(M, N, K, dtype, name, bias=(M + N) % 2 == 0, narrow=True)


# Rows, outputs, K, what the outputs are, and whether rows or columns are parted: products in two launches.
PARTS = [(4150, 2048, 3001, "bf16", False, "rows"), (4160, 4200, 1601, "bf16", False, "cols"), (4100, 2050, 1500, "fp32", False, "rows"),
         (2100, 4160, 1500, "fp32", False, "cols"), (4150, 1024, 3000, "bf16", True, "rows"), (4160, 2100, 1601, "bf16", True, "cols"),
         (2060, 2150, 1500, "fp32", True, "rows"), (2100, 2080, 1500, "fp32", True, "cols"), (2100, 2048, 2301, "f8", True, "rows"),
         (256, 16500, 2300, "f8", True, "cols")]


@pytest.mark.parametrize("M,N,K,kind,gated,part", PARTS)
def test_products_in_two_parts(M, N, K, kind, gated, part):
    dtype = {"bf16": BF16, "fp32": FP32, "f8": F8}[kind]
    for narrow in (False, True):
        if gated:
            check_gated(M, N, K, dtype, "silu", bias=True, narrow=narrow)
        else:
            check_matmul(M, N, K, dtype, bias=True, narrow=narrow)


def test_gated_outputs_that_are_given():
    from paper_2511_22009_amd import gated_matmul_f8
    g = gen(8)
    a, sa = P.codes(g, 70, 300)
    gate, sg = P.codes(g, 200, 300, 128, size=0.002)
    up, su = P.codes(g, 200, 300, 128, size=0.002)
    args = (a, sa, gate, sg, up, su)
    want, scale = gated_matmul_f8(*args, dtype=F8)
    room = torch.full((70, 240), 3.0, device="cuda").to(F8)
    scales = torch.full((70, 5), 4.0, device="cuda")
    q, s = gated_matmul_f8(*args, out=room[:, :200], out_scale=scales[:, 1:5:2])
    assert q.data_ptr() == room.data_ptr() and torch.equal(q.float(), want.float()) and torch.equal(s, scale)
    assert (room[:, 200:].float() == 3).all() and (scales[:, ::2] == 4).all()
    out = torch.empty((70, 200), device="cuda")
    assert gated_matmul_f8(*args, out=out) is out and torch.equal(out, gated_matmul_f8(*args, dtype=FP32))


def test_gated_block_of_zeros_and_of_nan():
    """A row of zeros leaves codes and scales 0; a NaN in a row all of its blocks NaN, the others as they were."""
    from paper_2511_22009_amd import gated_matmul_f8
    g = gen(9)
    a, sa = P.codes(g, 300, 256)
    gate, sg = P.codes(g, 300, 256, 128, size=0.002)
    up, su = P.codes(g, 300, 256, 128, size=0.002)
    want, scale = gated_matmul_f8(a, sa, gate, sg, up, su, dtype=F8)
    a.view(torch.uint8)[5] = 0
    a.view(torch.uint8)[200, 3] = 0x7f
    q, s = gated_matmul_f8(a, sa, gate, sg, up, su, dtype=F8)
    assert not q[5].float().any() and not s[5].any()
    assert torch.isnan(q[200].float()).all() and torch.isnan(s[200]).all()
    rest = [m for m in range(300) if m not in (5, 200)]
    assert torch.equal(q[rest].float(), want[rest].float()) and torch.equal(s[rest], scale[rest])


# ------------------------------------------------------------------------------- norms around a block

def make_rows(g, S, T, D, hd, yd, gate, mod, gains):
    h = (randn(g, S, T, D) * 2 + 0.3).to(hd)
    y = (randn(g, S, T, D) * torch.exp(randn(g, S, T, 1))).to(yd)
    v = dict(gate={"sample": lambda: randn(g, S, D), "channel": lambda: randn(g, D), None: lambda: None}[gate]())
    table = 0.3 * randn(g, S, 2 * D + 1)
    v["shift"], v["scale"] = (table[:, :D], table[:, D + 1:]) if mod else (None, None)
    v["post_gain"], v["pre_gain"] = (1 + 0.2 * randn(g, D), 1 + 0.2 * randn(g, D)) if gains else (None, None)
    return h, y, v


def check_rows(h, y, v, post, pre, r, dtype, eps=1e-6, **kw):
    from paper_2511_22009_amd import residual_norm
    ho, a = residual_norm(h, y, post=post, pre=pre, residual_scale=r, dtype=dtype, eps=eps, **v, **kw)
    want_h, eh, want, ea = P.residual_norm(h, y, v["gate"], post, v["post_gain"], r, pre, v["pre_gain"], v["scale"], v["shift"], eps)
    assert ho.dtype == h.dtype
    P.check(ho, want_h, eh, h.dtype)
    if dtype == F8:
        q, s = a
        assert q.dtype == F8 and q.shape == h.shape and s.shape == (*h.shape[:-1], P.blocks(h.shape[-1]))
        P.check_codes(q.flatten(0, -2), s.flatten(0, -2), want.flatten(0, -2), ea.flatten(0, -2))
    else:
        assert a.dtype == dtype
        P.check(a, want, ea, dtype)
    return ho, a


@pytest.mark.parametrize("dtype", [BF16, FP32, F8], ids=ids)
@pytest.mark.parametrize("S,T,D", [(1, 1, 1), (1, 1, 8), (8, 1, 1152), (3, 5, 7), (2, 9, 127), (1, 4, 128), (3, 2, 129), (2, 33, 256),
                                   (2, 3, 257), (3, 11, 768), (2, 5, 771), (1, 3, 1280), (2, 4, 1281), (1, 5, 2048), (2, 2, 2051),
                                   (1, 3, 4096), (2, 2, 8191), (1, 2, 16384)])
def test_residual_norm(S, T, D, dtype):
    g = gen(S * 100 + T * 10 + D)
    for n, (post, pre) in enumerate((("rms", "layer"), ("layer", "rms"), (None, "layer"), ("rms", "none"))):
        hd, yd = ((FP32, BF16), (BF16, FP32), (FP32, FP32), (BF16, BF16))[(n + D) % 4]
        h, y, v = make_rows(g, S, T, D, hd, yd, ("sample", "channel", None)[(n + T) % 3], n % 2 == 0, n != 3)
        check_rows(h, y, v, post, pre, (1.0, 0.5)[n % 2], dtype)


def test_residual_norm_many_rows():
    """More rows than workgroups at once, and samples that end inside a workgroup."""
    g = gen(20)
    for S, T, D in ((3, 3333, 64), (5, 1001, 770)):
        h, y, v = make_rows(g, S, T, D, FP32, BF16, "sample", True, True)
        check_rows(h, y, v, "rms", "layer", 1.0, BF16)
        check_rows(h, y, v, "layer", "rms", 1.0, F8)


def test_residual_norm_in_place_and_strides():
    from paper_2511_22009_amd import residual_norm
    g = gen(21)
    h, y, v = make_rows(g, 3, 40, 770, FP32, BF16, "sample", True, True)
    want = residual_norm(h, y, post="rms", pre="layer", **v)
    # rows inside wider ones, samples in another order, y transposed
    hs = torch.full((40, 3, 900), 7.0, device="cuda")
    view = hs[:, :, 5:775].transpose(0, 1)
    view.copy_(h)
    ys = y.transpose(0, 1).contiguous().transpose(0, 1)
    outs = torch.full((3, 40, 800), 7.0, device="cuda", dtype=BF16)
    ho, a = residual_norm(view, ys, post="rms", pre="layer", **v, h_out=view, out=outs[:, :, 1:771])
    assert ho is view and torch.equal(ho, want[0]) and torch.equal(a, want[1])
    assert (hs[:, :, :5] == 7).all() and (hs[:, :, 775:] == 7).all() and (outs[:, :, 0] == 7).all() and (outs[:, :, 771:] == 7).all()
    # codes into rows of their own
    want = residual_norm(h, y, post="rms", pre="layer", dtype=F8, **v)
    room = torch.full((3, 40, 800), 2.0, device="cuda").to(F8)
    scales = torch.full((3, 7, 41), 2.0, device="cuda")
    ho, (q, s) = residual_norm(h, y, post="rms", pre="layer", **v, out=room[:, :, :770], out_scale=scales[:, :, :40].transpose(1, 2))
    assert torch.equal(q.float(), want[1][0].float()) and torch.equal(s, want[1][1])
    assert (room[:, :, 770:].float() == 2).all() and (scales[:, :, 40] == 2).all()
    # two dims: one sample; no second output
    one = {k: (w if w is None or w.dim() == 1 else w[1]) for k, w in v.items()}
    flat = residual_norm(h[1], y[1], post="rms", pre="layer", **one)
    want = residual_norm(h, y, post="rms", pre="layer", **v)
    assert torch.equal(flat[0], want[0][1]) and torch.equal(flat[1], want[1][1])
    ho, none = residual_norm(h, y, post="rms", gate=v["gate"], post_gain=v["post_gain"])
    assert none is None and torch.equal(ho, want[0])


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e-22, 1e-12, 1e12, 1e25, 3e37])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_residual_norm_rows_of_every_size(size, kind, eps):
    """Rows whose squares, or sums, fp32 does not hold."""
    for D in (100, 1152, 5000):
        g = gen(D)
        y = ((randn(g, 1, 6, D) + 0.5).clamp(-3, 3) * size).float()
        h = torch.zeros_like(y)
        # far below eps the norm is the row divided by sqrt(eps): values that fp32 holds only as subnormal steps
        from paper_2511_22009_amd import residual_norm
        ho, a = residual_norm(h, y, post=kind, pre=kind, eps=eps, dtype=FP32)
        _, _, want, err = P.residual_norm(h, y, None, kind, None, 1.0, kind, None, None, None, eps)
        assert P.worst(a, want, err + want.abs() * P.U + 1e-35 / max(eps, 1e-30) ** 0.5 * (size < 1e-20) * (eps > 0)) <= 1.0


def test_residual_norm_rows_that_are_not_finite():
    """An infinity or a NaN stays in its row."""
    from paper_2511_22009_amd import residual_norm
    g = gen(23)
    h, y, v = make_rows(g, 2, 9, 300, FP32, BF16, "sample", True, True)
    want = residual_norm(h, y, post="rms", pre="layer", dtype=F8, **v)
    h[0, 3, 7], y[1, 8, 299] = float("inf"), float("nan")
    ho, (q, s) = residual_norm(h, y, post="rms", pre="layer", dtype=F8, **v)
    for n in range(2):
        for t in range(9):
            if (n, t) in ((0, 3), (1, 8)):
                assert torch.isnan(q[n, t].float()).all() and torch.isnan(s[n, t]).all()
            else:
                assert torch.equal(ho[n, t], want[0][n, t]) and torch.equal(q[n, t].float(), want[1][0][n, t].float())


# ------------------------------------------------------------------------------- together

def feed_forward(h, y, v, w, out):
    """The feed-forward half of a block as a program runs it."""
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, residual_norm
    S, T, D = h.shape
    h1, (a, sa) = residual_norm(h, y, gate=v["gate"], pre="layer", scale=v["scale"], shift=v["shift"], dtype=F8)
    g, sg = gated_matmul_f8(a.flatten(0, 1), sa.flatten(0, 1), *w["gate"], *w["up"], activation="silu", dtype=F8)
    z = matmul_f8(g, sg, *w["down"], w["bias"])
    h2, nxt = residual_norm(h1, z.view(S, T, D), gate=v["gate"], post="rms", post_gain=v["post_gain"], pre="layer", scale=v["scale"],
                            shift=v["shift"], dtype=out)
    return h1, (a, sa), (g, sg), z, h2, nxt


def make_block(g, S, T, D, F):
    from paper_2511_22009_amd import quantize_f8
    h, y, v = make_rows(g, S, T, D, FP32, BF16, "sample", True, True)
    w = {n: quantize_f8(randn(g, *s) / s[1] ** 0.5, block_rows=128) for n, s in (("gate", (F, D)), ("up", (F, D)), ("down", (D, F)))}
    w["bias"] = 0.1 * randn(g, D)
    return h, y, v, w


@pytest.mark.parametrize("S,T,D,F", [(1, 1, 96, 200), (3, 50, 192, 513), (2, 700, 768, 2048)])
def test_feed_forward(S, T, D, F):
    """Every step against 64 bits on what the step before left."""
    g = gen(D)
    h, y, v, w = make_block(g, S, T, D, F)
    h1, (a, sa), (q, sq), z, h2, nxt = feed_forward(h, y, v, w, BF16)
    want_h, eh, want, ea = P.residual_norm(h, y, v["gate"], None, None, 1.0, "layer", None, v["scale"], v["shift"], 1e-6)
    P.check(h1, want_h, eh, FP32)
    a, sa = a.flatten(0, 1), sa.flatten(0, 1)
    P.check_codes(a, sa, want.flatten(0, 1), ea.flatten(0, 1))
    want, err = P.gated(a, sa, *w["gate"], *w["up"], None, None, "silu", exact=True)
    P.check_codes(q, sq, want, err)
    want, err = P.product(q, sq, *w["down"], exact=False)
    want = want + w["bias"].double()
    P.check(z, want, err + (want.abs() + err) * P.U, BF16)
    want_h, eh, want, ea = P.residual_norm(h1, z.view(S, T, D), v["gate"], "rms", v["post_gain"], 1.0, "layer", None, v["scale"], v["shift"], 1e-6)
    P.check(h2, want_h, eh, FP32)
    P.check(nxt, want, ea, BF16)


def flat(x):
    for t in x:
        if isinstance(t, tuple):
            yield from flat(t)
        else:
            yield t.view(torch.uint8) if t.dtype == F8 else t


@pytest.mark.parametrize("S,T", [(1, 1), (2, 300)])
def test_feed_forward_in_a_graph(S, T):
    """Captured and replayed with new inputs, eager work between the replays: the eager bits."""
    g = gen(40)
    h, y, v, w = make_block(g, S, T, 256, 640)
    feed_forward(h, y, v, w, F8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = feed_forward(h, y, v, w, F8)
    for seed in range(3):
        new = make_rows(gen(50 + seed), S, T, 256, FP32, BF16, "sample", True, True)
        h.copy_(new[0])
        y.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        want = feed_forward(h, y, v, w, F8)
        torch.cuda.synchronize()
        for a, b in zip(flat(got), flat(want)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """The same chain on two streams, its calls in turn, many times over: the bits of one alone."""
    g = gen(42)
    blocks = [make_block(g, 2, 300, 256, 640), make_block(g, 1, 900, 384, 1000)]
    want = [[t.clone() for t in flat(feed_forward(*b, F8))] for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(6):
        for n, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[n].append(feed_forward(*blocks[n], F8))
    torch.cuda.synchronize()
    for n in range(2):
        for result in got[n]:
            for a, b in zip(flat(result), want[n]):
                assert torch.equal(a, b)


def test_feed_forward_on_a_stream():
    """Every call on a stream that is not the current one, its inputs dropped at once."""
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, quantize_f8, residual_norm
    g = gen(41)
    h, y, v, w = make_block(g, 2, 100, 256, 640)
    x = randn(g, 200, 256)
    want = [quantize_f8(x), *feed_forward(h, y, v, w, BF16)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    x2 = x.clone()
    s.wait_stream(torch.cuda.current_stream())
    a0 = quantize_f8(x2, stream=s)
    del x2
    h1, a = residual_norm(h, y, gate=v["gate"], pre="layer", scale=v["scale"], shift=v["shift"], dtype=F8, stream=s)
    q = gated_matmul_f8(a[0].flatten(0, 1), a[1].flatten(0, 1), *w["gate"], *w["up"], dtype=F8, stream=s)
    z = matmul_f8(*q, *w["down"], w["bias"], stream=s)
    h2, nxt = residual_norm(h1, z.view(2, 100, 256), gate=v["gate"], post="rms", post_gain=v["post_gain"], pre="layer", scale=v["scale"],
                            shift=v["shift"], stream=s)
    s.synchronize()
    for a, b in zip(flat([a0, h1, a, q, z, h2, nxt]), flat(want)):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------- refusals

def test_what_python_refuses():
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, quantize_f8, residual_norm
    g = gen(60)
    x = randn(g, 40, 300)
    a, sa = quantize_f8(x)
    b, sb = quantize_f8(randn(g, 200, 300), block_rows=128)
    for kw in (dict(block_rows=2), dict(out=a[:, :299]), dict(scale=sa[:, :2]), dict(scale=sa[:39]), dict(scale=sa[:, :1].expand(-1, 3))):
        with pytest.raises((ValueError, RuntimeError)):
            quantize_f8(x, **kw)
    for args in ((x, sa, b, sb), (a, sa.bfloat16(), b, sb), (a, sa, b.view(torch.int8), sb), (a, sa.cpu(), b, sb)):
        with pytest.raises(TypeError):
            matmul_f8(*args)
    for args in ((a, sa[:, :2], b, sb), (a, sb, b, sb), (a, sa, b, sa), (a, sa, b[:, :256], sb[:, :2]), (a[:, 1:], sa, b[:, 1:], sb),
                 (a.t(), sa, b, sb), (a[0], sa, b, sb)):
        with pytest.raises(ValueError):
            matmul_f8(*args)
    with pytest.raises(ValueError):
        matmul_f8(a, sa, b, sb, torch.zeros(199, device="cuda"))
    with pytest.raises(ValueError):
        matmul_f8(a, sa, b, sb, out=torch.empty((40, 199), device="cuda"))
    with pytest.raises(TypeError):
        matmul_f8(a, sa, b, sb, out=torch.empty((40, 208), device="cuda").to(F8)[:, :200])
    with pytest.raises(ValueError):
        gated_matmul_f8(a, sa, b, sb, b[:100], sb[:1])
    with pytest.raises(ValueError):
        gated_matmul_f8(a, sa, b, sb, b, sb, out_scale=torch.empty((40, 2), device="cuda"))
    with pytest.raises(ValueError):
        gated_matmul_f8(a, sa, b, sb, b, sb, out=torch.empty((40, 200), device="cuda").to(F8)[:, :200][:, ::1].t().contiguous().t())
    grad = torch.zeros((40, 300), device="cuda", requires_grad=True)
    for call in (lambda: quantize_f8(grad), lambda: residual_norm(grad, x), lambda: residual_norm(x, x, gate=grad[0])):
        with pytest.raises(TypeError, match="requires grad"):
            call()
    with torch.no_grad():
        quantize_f8(grad)
    h = randn(g, 2, 5, 300)
    for kw in (dict(y=h[:1]), dict(gate=torch.zeros(3, 300, device="cuda")), dict(gate=torch.zeros(299, device="cuda")),
               dict(post_gain=torch.zeros(2, 300, device="cuda")), dict(scale=torch.zeros(300, device="cuda")),
               dict(out=torch.empty_like(h)), dict(h_out=torch.empty_like(h)[:1]), dict(pre="rms", out_scale=torch.zeros(2, 5, 3, device="cuda")),
               dict(pre="rms", dtype=F8, out_scale=torch.zeros(2, 5, 2, device="cuda")),
               dict(pre="rms", out=torch.empty((2, 5, 300), device="cuda").to(F8))):
        with pytest.raises(ValueError):
            residual_norm(**{"h": h, "y": h, **kw})
    with pytest.raises(TypeError):
        residual_norm(h, h, h_out=h.bfloat16())
    from paper_2511_22009_amd import SFError
    for kw in (dict(h_out=h, y=h), dict(eps=-1.0), dict(residual_scale=float("inf")), dict(pre="rms", out=h), dict(h_out=h[:1].expand(2, -1, -1))):
        with pytest.raises(SFError):
            residual_norm(**{"h": h, "y": h + 1, **kw})


def test_empty_calls():
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, quantize_f8, residual_norm
    x = torch.zeros((0, 300), device="cuda")
    a, sa = quantize_f8(x)
    assert a.shape == (0, 300) and sa.shape == (0, 3)
    b, sb = quantize_f8(torch.ones((4, 300), device="cuda"), block_rows=128)
    assert matmul_f8(a, sa, b, sb).shape == (0, 4)
    none, scale = quantize_f8(x, block_rows=128)
    a, sa = quantize_f8(torch.ones((2, 300), device="cuda"))
    assert matmul_f8(a, sa, none, scale).shape == (2, 0)
    q, s = gated_matmul_f8(a, sa, none, scale, none, scale, dtype=F8)
    assert q.shape == (2, 0) and s.shape == (2, 0)
    h, out = residual_norm(torch.zeros((3, 0, 8), device="cuda"), torch.zeros((3, 0, 8), device="cuda"), pre="rms")
    assert h.shape == (3, 0, 8) and out.shape == (3, 0, 8)


def test_other_threads_run_while_a_call_is_under_way(tmp_path):
    """In the place of the library's entry points stands a function that waits (5 s at most) for what
    another Python thread does. Nothing is launched."""
    import ctypes
    import subprocess
    import threading

    from paper_2511_22009_amd import operators
    from test_gpu_operators_edges import WAITS
    src, lib = str(tmp_path / "w.cpp"), str(tmp_path / "w.so")
    with open(src, "w") as f:
        f.write(WAITS)
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", src, "-o", lib], check=True)
    w = ctypes.CDLL(lib)
    flag = ctypes.c_int.in_dll(w, "flag")
    x = randn(gen(107), 4, 256)
    a, sa = operators.quantize_f8(x)
    b, sb = operators.quantize_f8(x, block_rows=128)
    address = ctypes.cast(w.wait_for_flag, ctypes.c_void_p).value
    names = ("quantize_f8", "matmul_f8", "gated_matmul_f8", "residual_norm")
    entries = [ctypes.cast(getattr(operators.load_library(), "sf_" + n), ctypes.c_void_p).value for n in names]
    try:
        operators._ext.bind_f8(*[address] * 4)
        for call in (lambda: operators.quantize_f8(x), lambda: operators.matmul_f8(a, sa, b, sb),
                     lambda: operators.gated_matmul_f8(a, sa, b, sb, b, sb, dtype=F8), lambda: operators.residual_norm(x, x, pre="rms")):
            flag.value = 0
            setter = threading.Timer(0.02, lambda: setattr(flag, "value", 1))
            setter.start()
            call()                                     # SFError after 5 s if no other thread could run
            setter.join()
    finally:
        operators._ext.bind_f8(*entries)
    check_quantize(x, 1)                               # the library's own again
