"""Performance cases of the 8-bit projections and of the rotary queries and keys.

Each case is one call of an operator: the quantisation of token rows to 8-bit codes, the
matrix product of such codes, the rotation of heads by positions with several axes, and
the per-head norm of queries and keys with that rotation in the same pass. `listed()`
names the cases that are followed, `draw()` gives more of the same ranges, `prepare()`
builds what a program holds before the call, `run()` is the call (with `own`, the
framework's entry points; without, the operators' plain form in elementary torch
operations), `exact()` its result from the definition in 64-bit arithmetic.

Definitions:
  quantize  codes[m][k] = rint(127 x[m][k] / a[m]), ties to even, a[m] = max_k |x[m][k]|,
            scale[m] = a[m] / 127 in 32 bits; a row of zeros has codes and scale 0
  matmul    out[m][n] = sum_k A[m][k] B[n][k] * sa[m] * sb[n] + bias[n]
  rotate    pair j of a head, (x, y), turns by the angle p[axis_j] * freq_j of its token's
            position p: (x cos - y sin, x sin + y cos); dims of no pair stay
  qk        q and k are divided by sqrt(mean of squares over the head + eps), multiplied by
            a gain per dim and rotated
"""
import math

import torch

own = False

THETA, EPS = 10000.0, 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # ---- token rows to 8 bits
        # one row of the width-1152 networks: the launch and one row's latency
        {"name": "quant_one_row", "kind": "quantize", "M": 1, "K": 1152, "dtype": "bf16"},
        # the residual rows of a 640 x 368 picture with a queue of three, in 32 bits
        {"name": "quant_ragged_fp32", "kind": "quantize", "M": 2760, "K": 770, "dtype": "fp32"},
        # the MLP's hidden rows at 1024^2, four slots: bandwidth
        {"name": "quant_mlp_1024", "kind": "quantize", "M": 16384, "K": 4608, "dtype": "bf16"},
        # ---- products of 8-bit codes
        # one row against the QKV weights of the width-1152 networks: reads the weights once
        {"name": "mm_one_row", "kind": "matmul", "M": 1, "N": 3456, "K": 1152, "dtype": "bf16", "bias": True},
        # odd sizes in every direction, a long sum, 32-bit output, no bias
        {"name": "mm_odd_fp32", "kind": "matmul", "M": 1023, "N": 777, "K": 4321, "dtype": "fp32", "bias": False},
        # QKV at 512^2, four slots of 1024 tokens, width 768
        {"name": "mm_qkv_512", "kind": "matmul", "M": 4096, "N": 2304, "K": 768, "dtype": "bf16", "bias": True},
        # MLP up-projection at 1024^2, four slots of 4096 tokens, width 1152
        {"name": "mm_fc1_1024", "kind": "matmul", "M": 16384, "N": 4608, "K": 1152, "dtype": "bf16", "bias": True},
        # ---- rotary positions with several axes
        # queries of a short video clip: 8 frames of 30 x 52 patches, axes time, row, column
        {"name": "rot_video", "kind": "rotate", "rows": 1, "grid": "8,30,52", "heads": 16, "dh": 128, "dims": "16,56,56",
         "layout": "adjacent", "dtype": "bf16", "inverse": False, "shared": True, "far": 0.0},
        # keys of a small ragged picture turned back, in 32 bits, a part of each head only,
        # every row at positions of its own
        {"name": "rot_ragged_back", "kind": "rotate", "rows": 3, "grid": "10,14", "heads": 4, "dh": 48, "dims": "16,16",
         "layout": "axis_halves", "dtype": "fp32", "inverse": True, "shared": False, "far": 5000.0},
        # ---- norm and rotation of q and k in one pass
        # one new token for each of eight rows: latency
        {"name": "qk_one_token", "kind": "qk", "rows": 8, "grid": "1,1", "heads": 16, "kv_heads": 4, "dh": 128, "dims": "64,64",
         "layout": "halves", "dtype": "bf16", "packed": True, "shared": False, "far": 100000.0},
        # 512^2, four slots, width 768: q and k inside the packed QKV rows
        {"name": "qk_512", "kind": "qk", "rows": 4, "grid": "32,32", "heads": 12, "kv_heads": 12, "dh": 64, "dims": "32,32",
         "layout": "adjacent", "dtype": "bf16", "packed": True, "shared": True, "far": 0.0},
        # 1024^2, four slots, width 1152 (head dim 72), heads apart
        {"name": "qk_1024", "kind": "qk", "rows": 4, "grid": "64,64", "heads": 16, "kv_heads": 16, "dh": 72, "dims": "36,36",
         "layout": "halves", "dtype": "bf16", "packed": False, "shared": True, "far": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Rows from one to 32768, widths from 8 to 8192, tokens from one to 16384, head dims
    from 8 to 256 (odd multiples among them), one to four axes; below the work of the
    largest listed case of the kind."""
    kind = rng.choice(["quantize", "matmul", "matmul", "rotate", "qk", "qk"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    while kind == "quantize":
        c = {"kind": kind, "M": _log(rng, 1, 32768), "K": _log(rng, 8, 8192), "dtype": dtype}
        if c["M"] * c["K"] <= 16384 * 4608:
            return c
    while kind == "matmul":
        c = {"kind": kind, "M": _log(rng, 1, 32768), "N": _log(rng, 8, 8192), "K": _log(rng, 8, 8192), "dtype": dtype,
             "bias": rng.random() < 0.7}
        if rng.random() < 0.5:  # widths as networks have them
            c["N"], c["K"] = -(-c["N"] // 64) * 64, -(-c["K"] // 64) * 64
        if c["M"] * c["N"] * c["K"] <= 16384 * 4608 * 1152 and c["M"] * c["N"] <= 16384 * 4608:
            return c
    while True:
        axes = rng.randint(1, 4)
        n = _log(rng, 1, 16384)
        grid, left = [], n
        for a in range(axes - 1):
            side = max(1, min(left, _log(rng, 1, max(1, math.ceil(left ** (1.0 / (axes - a) * 1.5))))))
            grid.append(side)
            left = max(1, left // side)
        grid.append(left)
        dh = rng.choice([8, 32, 36, 48, 64, 64, 72, 80, 96, 98, 128, 128, 160, 256])
        part = rng.random() < 0.3 and dh >= 32
        pairs = (dh // 4 if part else dh // 2)
        cut = sorted(rng.randint(1, max(1, pairs - 1)) for _ in range(axes - 1))
        if rng.random() < 0.6:  # even shares, as networks have them
            cut = [pairs * (a + 1) // axes for a in range(axes - 1)]
        dims = [2 * (b - a) for a, b in zip([0] + cut, cut + [pairs])]
        heads = _log(rng, 1, 32)
        c = {"kind": kind, "rows": _log(rng, 1, 16), "grid": ",".join(map(str, grid)), "heads": heads, "dh": dh,
             "dims": ",".join(map(str, dims)), "layout": rng.choice(["adjacent", "halves", "axis_halves"]), "dtype": dtype,
             "shared": rng.random() < 0.5, "far": rng.choice([0.0, 0.0, 1000.0, 100000.0])}
        if kind == "rotate":
            c["inverse"] = rng.random() < 0.3
        else:
            c["kv_heads"] = rng.choice([h for h in (1, 2, 4, 8, heads) if heads % h == 0])
            c["packed"] = rng.random() < 0.5
        if c["rows"] * math.prod(grid) * (heads + c.get("kv_heads", 0)) * dh <= 16384 * 32 * 72:
            return c


# ------------------------------------------------------------------------- sizes

def _ints(text):
    return [int(v) for v in text.split(",")]


def _tokens(c):
    return math.prod(_ints(c["grid"]))


def work(c):
    """Every input read once and every output written once; the products of the sum."""
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "quantize":
        M, K = c["M"], c["K"]
        return {"bytes": float(M * K * (es + 1) + 4 * M), "flops": 3.0 * M * K}
    if c["kind"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": float((M + N) * K + es * M * N + 4 * (M + N) + 4 * N * c["bias"]), "flops": 2.0 * M * N * K}
    T, heads = c["rows"] * _tokens(c), c["heads"] + c.get("kv_heads", 0)
    pos = 4 * len(_ints(c["dims"])) * (_tokens(c) if c["shared"] else T)
    return {"bytes": float(2 * es * T * heads * c["dh"] + pos), "flops": (7.0 if c["kind"] == "qk" else 3.0) * T * heads * c["dh"]}


# ------------------------------------------------------------------------ inputs

def _codes(g, rows, K):
    """8-bit codes as a quantisation leaves them (a bell with its largest at 127), the rows
    at a pitch of a multiple of 16 bytes, and the scales of the rows."""
    pitch = -(-K // 16) * 16
    q = torch.zeros((rows, pitch), dtype=torch.int8, device="cuda")
    q[:, :K] = (torch.randn((rows, K), generator=g, device="cuda") * 36).round().clamp(-127, 127).to(torch.int8)
    s = torch.exp(torch.randn(rows, generator=g, device="cuda") * 0.5) * 0.02
    return q[:, :K], s


def _freqs(dims):
    """Frequency of every pair: theta^(-2 i / d) for pair i of an axis of d dims."""
    return [THETA ** (-2.0 * i / d) for d in dims for i in range(d // 2)]


def _pairs(c):
    """The two dims of every pair, and its axis."""
    dims = _ints(c["dims"])
    P = sum(dims) // 2
    axis = [a for a, d in enumerate(dims) for _ in range(d // 2)]
    if c["layout"] == "adjacent":
        lo = [2 * j for j in range(P)]
        hi = [2 * j + 1 for j in range(P)]
    elif c["layout"] == "halves":
        lo = list(range(P))
        hi = [j + P for j in range(P)]
    else:
        lo, hi, base = [], [], 0
        for d in dims:
            lo += [base + i for i in range(d // 2)]
            hi += [base + d // 2 + i for i in range(d // 2)]
            base += d
    return lo, hi, axis


def _positions(c, g):
    """[rows or 1][tokens][axes]: the token's place in the grid, moved per row by up to
    `far` (a clip's place in a long one, a tile's in a large picture)."""
    grid = _ints(c["grid"])
    axes = torch.meshgrid(*[torch.arange(n, dtype=torch.float32, device="cuda") for n in grid], indexing="ij")
    p = torch.stack([a.reshape(-1) for a in axes], 1)[None]
    rows = 1 if c["shared"] else c["rows"]
    at = torch.floor(torch.rand((rows, 1, len(grid)), generator=g, device="cuda") * (c["far"] + (0 if c["shared"] else 1)))
    return (p + at).contiguous()


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 41)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] == "quantize":
        M, K = c["M"], c["K"]
        x = torch.randn((M, K), generator=g, device="cuda")
        # a few channels far larger than the rest, as activations have them; rows of
        # different size; some rows of padding, all zero
        wide = torch.rand(K, generator=g, device="cuda") < 0.01
        x *= torch.where(wide, 20.0, 1.0) * torch.exp(torch.randn((M, 1), generator=g, device="cuda"))
        if M > 8:
            x[torch.rand(M, generator=g, device="cuda") < 0.02] = 0.0
        s["x"] = x.to(dt)
    elif c["kind"] == "matmul":
        s["a"], s["a_scale"] = _codes(g, c["M"], c["K"])
        s["b"], s["b_scale"] = _codes(g, c["N"], c["K"])
        s["bias"] = torch.randn(c["N"], generator=g, device="cuda") if c["bias"] else None
    else:
        R, T, H, dh = c["rows"], _tokens(c), c["heads"], c["dh"]
        s["pos"] = _positions(c, g)
        if c["kind"] == "rotate":
            s["x"] = torch.randn((R, T, H, dh), generator=g, device="cuda").to(dt)
        else:
            Hk = c["kv_heads"]
            if c["packed"]:  # rows of q, k and v heads, as one projection leaves them
                qkv = (torch.randn((R, T, H + 2 * Hk, dh), generator=g, device="cuda") * 3).to(dt)
                s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + Hk]
            else:  # [rows][heads][tokens][dh], as attention reads them
                s["q"] = (torch.randn((R, H, T, dh), generator=g, device="cuda") * 3).to(dt).transpose(1, 2)
                s["k"] = (torch.randn((R, Hk, T, dh), generator=g, device="cuda") * 3).to(dt).transpose(1, 2)
            s["q_gain"] = 1.0 + 0.2 * torch.randn(dh, generator=g, device="cuda")
            s["k_gain"] = 1.0 + 0.2 * torch.randn(dh, generator=g, device="cuda")
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if c["kind"] in ("rotate", "qk"):
        # the plan of the rotation: a program makes it once for its network
        lo, hi, axis = _pairs(c)
        s["lo"], s["hi"], s["axis"] = (torch.tensor(v, device="cuda") for v in (lo, hi, axis))
        s["freq"] = torch.tensor(_freqs(_ints(c["dims"])), dtype=torch.float64, device="cuda")
        if own:
            from paper_2511_22009_amd import Rotary
            s["rotary"] = Rotary(_ints(c["dims"]), theta=THETA, layout=c["layout"])
    return s


def _turn(x, s, inverse=False):
    """x [rows][tokens][heads][dh] in 32 bits, turned; angles in 64 bits, as far positions
    need them, their cosines and sines in 32."""
    angle = (s["pos"].double()[:, :, s["axis"]] * s["freq"])[:, :, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if inverse:
        sin = -sin
    a, b = x[..., s["lo"]], x[..., s["hi"]]
    out = x.clone()
    out[..., s["lo"]] = a * cos - b * sin
    out[..., s["hi"]] = a * sin + b * cos
    return out


def _norm(x, gain):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain


def run(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "quantize":
        if own:
            from paper_2511_22009_amd import quantize_rows
            codes, scale = quantize_rows(s["x"])
        else:
            x = s["x"].float()
            a = x.abs().amax(1)
            scale = a / 127.0
            # in 64 bits: quotients next to a half
            codes = torch.round(x.double() * 127.0 / torch.where(a > 0, a, 1.0).double()[:, None]).to(torch.int8)
        return {"codes": codes, "scale": scale}
    if c["kind"] == "matmul":
        if own:
            from paper_2511_22009_amd import matmul_i8
            return matmul_i8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], dtype=dt)
        out = s["a"].float() @ s["b"].float().t()
        out = out * s["a_scale"][:, None] * s["b_scale"]
        return (out if s["bias"] is None else out + s["bias"]).to(dt)
    if c["kind"] == "rotate":
        if own:
            from paper_2511_22009_amd import rotate
            return rotate(s["x"], s["pos"], s["rotary"], inverse=c["inverse"])
        return _turn(s["x"].float(), s, c["inverse"]).to(dt)
    if own:
        from paper_2511_22009_amd import qk_norm_rotate
        return qk_norm_rotate(s["q"], s["k"], s["q_gain"], s["k_gain"], s["pos"], s["rotary"], eps=EPS)
    return _turn(_norm(s["q"], s["q_gain"]), s).to(dt), _turn(_norm(s["k"], s["k_gain"]), s).to(dt)


# ----------------------------------------------------------------- 64-bit results

def _turned(x, c, pos, inverse):
    """Each pair as a complex number times e^(i angle)."""
    lo, hi, axis = _pairs(c)
    out = x.clone()
    for j, f in enumerate(_freqs(_ints(c["dims"]))):
        w = torch.polar(torch.ones_like(pos[:, :, 0]), pos[:, :, axis[j]] * (-f if inverse else f))[:, :, None]
        z = torch.complex(x[..., lo[j]].contiguous(), x[..., hi[j]].contiguous()) * w
        out[..., lo[j]], out[..., hi[j]] = z.real, z.imag
    return out


def exact(c, seed):
    s = _inputs(c, seed)
    if c["kind"] == "quantize":
        return {"codes": None, "scale": s["x"].double().abs().amax(1) / 127.0}
    if c["kind"] == "matmul":
        out = (s["a"].double() * s["a_scale"].double()[:, None]) @ (s["b"].double() * s["b_scale"].double()[:, None]).t()
        return out if s["bias"] is None else out + s["bias"].double()
    pos = s["pos"].double()
    if c["kind"] == "rotate":
        return _turned(s["x"].double(), c, pos, c["inverse"])
    both = []
    for n in ("q", "k"):
        x = s[n].double()
        size = torch.sqrt(x.square().sum(-1, keepdim=True) / c["dh"] + EPS)
        both.append(_turned(x / size * s[n + "_gain"].double(), c, pos, False))
    return tuple(both)
