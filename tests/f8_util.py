"""Plain 64-bit forms of the 8-bit floating point operators, and what roundings may add up to."""
import math

import torch

F8, BF16, FP32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}   # half a step of the type, relative
U = 2.0 ** -24
BLOCK, TOP = 128, 448.0


def gen(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def randn(g, *shape, dtype=FP32):
    return torch.randn(shape, generator=g, device=g.device).to(dtype)


def blocks(n):
    return -(-n // BLOCK)


def nearest_f8(q):
    """The e4m3 number nearest to q (64 bits), ties to even, at most 448."""
    e = torch.frexp(q).exponent.clamp_min(-5) - 4
    step = ((e + 1023).to(torch.int64) << 52).view(torch.float64)  # 2^e, every bit of it
    return (torch.round(q / step) * step).clamp(-TOP, TOP)


def tops(x, block_rows=1):
    """Largest magnitude of every block, [blocks of rows, blocks of columns]."""
    M, K = x.shape
    mb = -(-M // block_rows)
    x = torch.nn.functional.pad(x.double().abs(), (0, blocks(K) * BLOCK - K, 0, mb * block_rows - M))
    return x.view(mb, block_rows, blocks(K), BLOCK).amax((1, 3))


def spread(scale, M, K, block_rows=1):
    """A block's number for every one of its values."""
    return scale.repeat_interleave(block_rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]


def plain_quantize(x, block_rows=1):
    """Codes (as 64-bit values) and fp32 scales from the definition; the quotient of two fp32 numbers in 64 bits lies
    on the exact one's side of every tie, and top / 448 in 64 bits, a number of sevenths of a step, is no tie of fp32."""
    scale = (tops(x, block_rows) / TOP).float()
    s = spread(scale.double(), *x.shape, block_rows)
    return torch.where(s > 0, nearest_f8(x.double() / torch.where(s > 0, s, 1.0)), 0.0), scale


def values(codes, scale, block_rows=1):
    return codes.double() * spread(scale.double(), *codes.shape, block_rows)


def codes(g, rows, K, block_rows=1, size=0.002, pitch=None):
    """Codes as a quantisation leaves them, NaN behind K where the rows have room, and scales."""
    ld = -(-K // 16) * 16 if pitch is None else pitch
    q = torch.full((rows, ld), float("nan"), device=g.device).to(F8)
    q[:, :K] = (torch.randn((rows, K), generator=g, device=g.device) * 130).clamp(-TOP, TOP).to(F8)
    s = torch.exp(torch.randn((blocks(K), -(-rows // block_rows)), generator=g, device=g.device) * 0.5) * size
    return q[:, :K], s.t()


def narrow(q):
    """Codes of magnitudes 1 to 3.75 only: their products are multiples of 2^-6 with powers of two from 1 to 4, so that none
    is cut off below 2^-13 of the largest one's, and a block's sum is exact in fp32."""
    q.view(torch.uint8).bitwise_and_(0x8f).add_(0x38)
    return q


def cut_off(a, sa, b, sb):
    """What the matrix cores may leave out of sums of codes: of every eight adjacent products all but the largest lose less
    than 2^-13 of its power of two each. (Products eight apart are added in fp32.)"""
    x, w = values(a, sa).abs(), values(b, sb, BLOCK).abs()
    total = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device=x.device)
    for k in range(0, x.shape[1], 8):
        total += (x[:, None, k:k + 8] * w[None, :, k:k + 8]).amax(2)
    return total * 7 * 2.0 ** -13


def product(a, sa, b, sb, exact):
    """The product in 64 bits and how far fp32 sums may be from it: 128 additions of a block on the matrix
    cores, each off by at most a step (they need not round to nearest), then per block the scales'
    product, one fma and the sums' own error; where the sums are not `exact`, what they cut off."""
    x, w = values(a, sa), values(b, sb, BLOCK)
    total = x.abs() @ w.abs().t()
    err = total * (BLOCK * 2 * U + (blocks(a.shape[1]) + 2) * U)
    return x @ w.t(), err if exact else err + cut_off(a, sa, b, sb)


def worst(got, want, allowed):
    """Largest |got - want| / allowed (0 where both are 0)."""
    got = got.double()
    assert got.shape == want.shape and torch.isfinite(got).all()
    return float(((got - want).abs() / allowed.clamp_min(1e-300)).max()) if got.numel() else 0.0


def check(got, want, err, dtype):
    assert worst(got, want, err + HALF[dtype] * (want.abs() + err)) <= 1.0


def check_codes(q, scale, want, err):
    """Codes and scales [rows, blocks] of values `want`, computed to within `err`: the scale is a step of the block's
    largest, a code at most half a step of e4m3 off (2^-4 of a value, 2^-10 of the scale's unit below
    the normal codes) and may fall on the other side of a tie, which `err` counts."""
    M, K = want.shape
    top, top_err = tops(want), tops(err)
    assert worst(scale, top / TOP, top_err / TOP + top / TOP * 2 * U) <= 1.0
    s = spread(scale.double(), M, K)
    # a code's half step is that of the binade it rounds into; the largest code is never passed by more than err
    allowed = err + (want.abs() + err) * 2.0 ** -4 + s * 2.0 ** -10 + want.abs() * 4 * U
    assert worst(values(q, scale), want, allowed) <= 1.0


def act(x, name):
    """The activation in 64 bits, and its relative error in fp32 with the hardware's exp2 and reciprocal (a step each):
    an error of the exponent y counts |y| times."""
    if name == "silu":
        return x * torch.sigmoid(x), (8 + 4 * x.abs()) * U
    y = math.sqrt(8.0 / math.pi) * (x + 0.044715 * x ** 3)
    return x * torch.sigmoid(y), (8 + 8 * y.abs()) * U


def gated(a, sa, gate, sg, up, su, gate_bias, up_bias, name, exact):
    """act(G) U in 64 bits and how far fp32 may be: |act'| is below 1.13 for both activations."""
    g, eg = product(a, sa, gate, sg, exact)
    u, eu = product(a, sa, up, su, exact)
    if gate_bias is not None:
        g = g + gate_bias.double()
        eg = eg + (g.abs() + eg) * U
    if up_bias is not None:
        u = u + up_bias.double()
        eu = eu + (u.abs() + eu) * U
    f, rel = act(g, name)
    ef = 1.13 * eg + (f.abs() + 1.13 * eg) * rel + 1e-37
    return f * u, ef * (u.abs() + eu) + f.abs() * eu + (f * u).abs() * 2 * U


def norm(x, err, kind, gain, eps):
    """The norm in 64 bits and how far fp32 may be, for x that is off by at most err. Sums of D terms in pieces of four
    over 64 or 256 lanes: at most D / 64 + 12 roundings of a partial sum."""
    if kind in (None, "none"):
        return x, err  # the gain belongs to the norm's caller here
    D = x.shape[-1]
    sums = (D / 64 + 12) * U
    if kind == "layer":
        err = err + err.mean(-1, keepdim=True) + x.abs().mean(-1, keepdim=True) * sums + x.abs() * U
        x = x - x.mean(-1, keepdim=True)
    by = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x * by
    return n, by * err + n.abs() * (by * err.square().mean(-1, keepdim=True).sqrt() + sums + 6 * U)


def residual_norm(h, y, gate, post, post_gain, r, pre, pre_gain, scale, shift, eps):
    """(h', its error, a, its error) in 64 bits; vectors are [dims] or [samples, dims]."""
    h, y = h.double(), y.double()

    def vec(v, other):
        if v is None:
            return torch.tensor(other, dtype=torch.float64, device=h.device)
        v = v.double()
        return v[:, None] if v.dim() == 2 and h.dim() == 3 else v

    u, eu = norm(y, torch.zeros_like(y), post, None, eps)
    by = vec(gate, 1.0) * vec(post_gain, 1.0)
    out = float(r) * h + by * u
    eo = by.abs() * (eu + u.abs() * 3 * U) + out.abs() * U
    n, en = norm(out, eo, pre, None, eps)
    by = vec(pre_gain, 1.0) * (1.0 + vec(scale, 0.0))
    a = n * by + vec(shift, 0.0)
    # the gain and the factor with scale are applied one after the other, 1 + scale unrounded
    g = vec(pre_gain, 1.0).abs() * (1.0 + vec(scale, 0.0).abs())
    return out, eo, a, g * (en + n.abs() * 4 * U) + a.abs() * 2 * U
