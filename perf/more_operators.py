"""Performance cases of a block's feed-forward half in 8-bit floating point.

Each case is one call of an operator: the quantisation of rows or weights to e4m3 codes with
a scale per block of 128, the matrix product of such codes, the two projections of a gated
feed-forward with their activation and product, and the norms after and before a block with
its gate and residual. `listed()` names the cases that are followed, `draw()` gives more of
the same ranges, `prepare()` builds what a program holds before the call, `run()` is the
call (with `own`, the framework's entry points; without, the operators' plain form in
elementary torch operations), `exact()` its result from the definition in 64-bit arithmetic.

Definitions (blocks of 128 columns, the last one as long as what is left):
  quantize  per block of 1 or 128 rows: s = max |x| / 448 in 32 bits, code = the e4m3 number
            nearest to x / s, ties to even; a block of zeros has codes and scale 0
  matmul    out[m][n] = sum over blocks b of (sum_k in b A[m][k] B[n][k]) sa[m][b] sb[n / 128][b] + bias[n]
  gated     out = act(A Wg^T + bg) (A Wu^T + bu), both products as above, act silu or tanh-GELU; as
            values, or as codes with a scale per row and block of 128 outputs
  norms     h' = r h + gate post(y) post_gain, a = pre(h') pre_gain (1 + scale) + shift, of
            every row; a norm divides by the root mean square ("rms"), or takes the mean off
            and divides by the deviation ("layer"), or is none; a as values or as codes
"""
import math

import torch

own = False

EPS, BLOCK, TOP = 1e-6, 128, 448.0
F8 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "f8": F8}
SIZE = {"bf16": 2, "fp32": 4, "f8": 1}


def listed():
    return [
        # ---- to codes
        # one row of the width-1152 networks: the launch and one row's latency
        {"name": "f8_quant_one_row", "kind": "quantize", "M": 1, "K": 1152, "dtype": "bf16", "block": 1},
        # weights of an MLP as they are loaded, in 32 bits
        {"name": "f8_quant_weights", "kind": "quantize", "M": 4608, "K": 1152, "dtype": "fp32", "block": 128},
        # attention outputs at 1024^2, four slots, width 1152: bandwidth
        {"name": "f8_quant_1024", "kind": "quantize", "M": 16384, "K": 1152, "dtype": "bf16", "block": 1},
        # ---- products
        # one row against the QKV weights of the width-1152 networks: reads the weights once
        {"name": "f8_mm_one_row", "kind": "matmul", "M": 1, "N": 3456, "K": 1152, "dtype": "bf16", "bias": True},
        # odd sizes in every direction, a long sum, 32-bit output, no bias
        {"name": "f8_mm_odd_fp32", "kind": "matmul", "M": 517, "N": 1001, "K": 4321, "dtype": "fp32", "bias": False},
        # MLP down-projection at 1024^2, four slots of 4096 tokens, width 1152
        {"name": "f8_mm_down_1024", "kind": "matmul", "M": 16384, "N": 1152, "K": 4608, "dtype": "bf16", "bias": True},
        # ---- gated projections
        # the conditioning's eight rows through a gated MLP: both weights once
        {"name": "f8_gated_few", "kind": "gated", "M": 8, "F": 2048, "K": 768, "dtype": "bf16", "bias": True, "act": "silu"},
        # 512^2, four slots, width 768, outputs as values
        {"name": "f8_gated_512", "kind": "gated", "M": 4096, "F": 2048, "K": 768, "dtype": "bf16", "bias": False, "act": "gelu"},
        # 1024^2, four slots, width 1152, outputs as the codes that the down-projection reads
        {"name": "f8_gated_1024", "kind": "gated", "M": 16384, "F": 4608, "K": 1152, "dtype": "f8", "bias": False, "act": "silu"},
        # ---- norms after and before a block
        # one token for each of eight slots: latency
        {"name": "norms_one_token", "kind": "norms", "S": 8, "T": 1, "D": 1152, "h": "fp32", "y": "bf16", "dtype": "bf16",
         "post": "rms", "pre": "layer", "gate": "sample", "mod": True, "gains": True, "r": 1.0},
        # a queue of three at 640 x 368, odd width, everything in 32 bits, a gate per channel
        {"name": "norms_ragged_fp32", "kind": "norms", "S": 3, "T": 920, "D": 771, "h": "fp32", "y": "fp32", "dtype": "fp32",
         "post": "layer", "pre": "rms", "gate": "channel", "mod": False, "gains": True, "r": 0.5},
        # 1024^2, four slots, width 1152, the next block's input as codes: bandwidth
        {"name": "norms_1024", "kind": "norms", "S": 4, "T": 4096, "D": 1152, "h": "fp32", "y": "bf16", "dtype": "f8",
         "post": "rms", "pre": "layer", "gate": "sample", "mod": True, "gains": True, "r": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Rows from one to 32768, widths from 8 to 8192, tokens from one to 16384 in one to 16
    slots, odd sizes among them; below the work of the largest listed case of the kind."""
    kind = rng.choice(["quantize", "matmul", "matmul", "gated", "gated", "norms", "norms"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    while kind == "quantize":
        c = {"kind": kind, "M": _log(rng, 1, 32768), "K": _log(rng, 8, 8192), "dtype": dtype, "block": rng.choice([1, 1, 128])}
        if c["M"] * c["K"] <= 16384 * 1152:
            return c
    wide = rng.random() < 0.5  # widths as networks have them
    while kind == "matmul":
        c = {"kind": kind, "M": _log(rng, 1, 32768), "N": _log(rng, 8, 8192), "K": _log(rng, 8, 8192), "dtype": dtype,
             "bias": rng.random() < 0.7}
        if wide:
            c["N"], c["K"] = -(-c["N"] // 64) * 64, -(-c["K"] // 64) * 64
        if c["M"] * c["N"] * c["K"] <= 16384 * 4608 * 1152 and c["M"] * c["N"] <= 16384 * 1152:
            return c
    while kind == "gated":
        c = {"kind": kind, "M": _log(rng, 1, 32768), "F": _log(rng, 8, 8192), "K": _log(rng, 8, 4096),
             "dtype": rng.choice([dtype, "f8"]), "bias": rng.random() < 0.5, "act": rng.choice(["silu", "gelu"])}
        if wide:
            c["F"], c["K"] = -(-c["F"] // 64) * 64, -(-c["K"] // 64) * 64
        if c["M"] * c["F"] * c["K"] <= 16384 * 4608 * 1152 and c["M"] * c["F"] <= 16384 * 1152:
            return c
    while True:
        c = {"kind": kind, "S": _log(rng, 1, 16), "T": _log(rng, 1, 16384), "D": _log(rng, 8, 8192),
             "h": rng.choice(["fp32", "fp32", "bf16"]), "y": rng.choice(["bf16", "bf16", "fp32"]),
             "dtype": rng.choice(["bf16", "f8", "fp32"]), "post": rng.choice(["rms", "rms", "layer", "none"]),
             "pre": rng.choice(["layer", "layer", "rms"]), "gate": rng.choice(["sample", "sample", "channel", "none"]),
             "mod": rng.random() < 0.7, "gains": rng.random() < 0.7, "r": rng.choice([1.0, 0.5])}
        if wide:
            c["D"] = -(-c["D"] // 64) * 64
        if c["S"] * c["T"] * c["D"] * (2 * SIZE[c["h"]] + SIZE[c["y"]] + SIZE[c["dtype"]]) <= 16384 * 1152 * 11:
            return c


# ------------------------------------------------------------------------- sizes

def _up(n, to):
    return -(-n // to) * to


def _blocks(n):
    return -(-n // BLOCK)


def work(c):
    """Every input read once and every output written once; the products of the sums."""
    es = SIZE[c["dtype"]]
    if c["kind"] == "quantize":
        M, K = c["M"], c["K"]
        return {"bytes": float(M * K * (es + 1) + 4 * -(-M // c["block"]) * _blocks(K)), "flops": 2.0 * M * K}
    if c["kind"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        scales = 4 * (M + _blocks(N)) * _blocks(K)
        return {"bytes": float((M + N) * K + scales + es * M * N + 4 * N * c["bias"]), "flops": 2.0 * M * N * K}
    if c["kind"] == "gated":
        M, F, K = c["M"], c["F"], c["K"]
        scales = 4 * (M + 2 * _blocks(F)) * _blocks(K) + 4 * M * _blocks(F) * (c["dtype"] == "f8")
        return {"bytes": float((M + 2 * F) * K + scales + es * M * F + 8 * F * c["bias"]), "flops": 4.0 * M * F * K}
    rows, D = c["S"] * c["T"], c["D"]
    vectors = D * ({"sample": c["S"], "channel": 1, "none": 0}[c["gate"]] + 2 * c["S"] * c["mod"] + c["gains"] * (1 + (c["post"] != "none")))
    scales = 4 * rows * _blocks(D) * (c["dtype"] == "f8")
    return {"bytes": float(rows * D * (2 * SIZE[c["h"]] + SIZE[c["y"]] + es) + 4 * vectors + scales), "flops": 12.0 * rows * D}


# ------------------------------------------------------------------------ inputs

def _codes(g, rows, K, block):
    """Codes as a quantisation leaves them (a bell, its largest at the type's), the rows at a
    pitch of a multiple of 16 bytes, and the blocks' scales, adjacent along the rows."""
    pitch = _up(K, 16 if K < 1024 else 128)
    q = torch.zeros((rows, pitch), dtype=F8, device="cuda")
    q[:, :K] = (torch.randn((rows, K), generator=g, device="cuda") * 130).clamp(-TOP, TOP).to(F8)
    s = torch.exp(torch.randn((_blocks(K), -(-rows // block)), generator=g, device="cuda") * 0.5) * 0.002
    return q[:, :K], s.t()


def _bias(g, n, wanted):
    return torch.randn(n, generator=g, device="cuda") if wanted else None


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 43)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["kind"] == "quantize":
        M, K = c["M"], c["K"]
        x = rand(M, K)
        # a few channels far larger than the rest, as activations have them; rows of
        # different size; some rows of padding, all zero
        wide = torch.rand(K, generator=g, device="cuda") < 0.01
        x *= torch.where(wide, 20.0, 1.0) * torch.exp(rand(M, 1))
        if M > 8:
            x[torch.rand(M, generator=g, device="cuda") < 0.02] = 0.0
        s["x"] = x.to(DTYPES[c["dtype"]])
    elif c["kind"] == "matmul":
        s["a"], s["a_scale"] = _codes(g, c["M"], c["K"], 1)
        s["b"], s["b_scale"] = _codes(g, c["N"], c["K"], BLOCK)
        s["bias"] = _bias(g, c["N"], c["bias"])
    elif c["kind"] == "gated":
        s["a"], s["a_scale"] = _codes(g, c["M"], c["K"], 1)
        # projections of a size that the activation's bend sees
        for n in ("gate", "up"):
            s[n], scale = _codes(g, c["F"], c["K"], BLOCK)
            s[n + "_scale"] = (scale * (15.0 / math.sqrt(c["K"]))).t().contiguous().t()
            s[n + "_bias"] = _bias(g, c["F"], c["bias"])
    else:
        S, T, D = c["S"], c["T"], c["D"]
        # a residual stream of a few times the block's output, some channels far larger
        wide = torch.where(torch.rand(D, generator=g, device="cuda") < 0.01, 15.0, 1.0)
        s["h"] = (rand(S, T, D) * 2 * wide + 0.3).to(DTYPES[c["h"]])
        s["y"] = (rand(S, T, D) * wide).to(DTYPES[c["y"]])
        s["gate"] = {"sample": rand(S, D), "channel": rand(D), "none": None}[c["gate"]]
        # one table of the conditioning holds both, so samples are 2 D apart
        table = 0.3 * rand(S, 2 * D)
        s["shift"], s["scale"] = (table[:, :D], table[:, D:]) if c["mod"] else (None, None)
        s["post_gain"] = 1.0 + 0.2 * rand(D) if c["gains"] and c["post"] != "none" else None
        s["pre_gain"] = 1.0 + 0.2 * rand(D) if c["gains"] else None
    return s


# -------------------------------------------------------------------- plain form

def _nearest_f8(q):
    """The e4m3 number nearest to q (64 bits), ties to even: a step is 2^-3 of the binade, 2^-9 at least."""
    e = torch.frexp(q).exponent.clamp_min(-5) - 4
    step = ((e + 1023).to(torch.int64) << 52).view(torch.float64)  # 2^e, every bit of it
    return (torch.round(q / step) * step).float().to(F8)


def _to_codes(x, block):
    """Codes of x (32 bits) and the scales [blocks of rows][blocks of columns]; quotients in 64 bits, as
    those next to a tie need."""
    M, K = x.shape
    mb, kb = -(-M // block), _blocks(K)
    padded = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, mb * block - M)).view(mb, block, kb, BLOCK)
    scale = (padded.abs().amax((1, 3)).double() / TOP).float()
    q = padded.double() / torch.where(scale > 0, scale, 1.0).double()[:, None, :, None]
    return _nearest_f8(q).view(mb * block, kb * BLOCK)[:M, :K], scale


def _values(q, scale, block, dtype):
    """What codes with their scales stand for."""
    rows = scale.to(dtype).repeat_interleave(block, 0)[:q.shape[0]]
    return q.to(dtype) * rows.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _act(x, name):
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _norm(x, kind, gain):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x if gain is None else x * gain


def _per_sample(v):
    """[samples][D] against [samples][tokens][D]; one for all stays."""
    return v[:, None] if v is not None and v.dim() == 2 else v


def _norms(h, y, gate, post_gain, pre_gain, scale, shift, c):
    u = _norm(y, c["post"], post_gain)
    h = c["r"] * h + (u if gate is None else _per_sample(gate) * u)
    a = _norm(h, c["pre"], pre_gain)
    return h, a if scale is None else a * (1.0 + _per_sample(scale)) + _per_sample(shift)


def run(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "quantize":
        if own:
            from paper_2511_22009_amd import quantize_f8
            codes, scale = quantize_f8(s["x"], block_rows=c["block"])
        else:
            codes, scale = _to_codes(s["x"].float(), c["block"])
        return {"codes": codes, "scale": scale}
    if c["kind"] == "matmul":
        if own:
            from paper_2511_22009_amd import matmul_f8
            return matmul_f8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], dtype=dt)
        out = _values(s["a"], s["a_scale"], 1, torch.float32) @ _values(s["b"], s["b_scale"], BLOCK, torch.float32).t()
        return (out if s["bias"] is None else out + s["bias"]).to(dt)
    if c["kind"] == "gated":
        if own:
            from paper_2511_22009_amd import gated_matmul_f8
            out = gated_matmul_f8(s["a"], s["a_scale"], s["gate"], s["gate_scale"], s["up"], s["up_scale"], s["gate_bias"],
                                  s["up_bias"], activation="silu" if c["act"] == "silu" else "gelu_tanh", dtype=dt)
        else:
            a = _values(s["a"], s["a_scale"], 1, torch.float32)
            g = a @ _values(s["gate"], s["gate_scale"], BLOCK, torch.float32).t()
            u = a @ _values(s["up"], s["up_scale"], BLOCK, torch.float32).t()
            if c["bias"]:
                g, u = g + s["gate_bias"], u + s["up_bias"]
            out = _act(g, c["act"]) * u
            out = _to_codes(out, 1) if dt == F8 else out.to(dt)
        return {"codes": out[0], "scale": out[1]} if dt == F8 else out
    if own:
        from paper_2511_22009_amd import residual_norm
        kind = {"none": None}
        h, out = residual_norm(s["h"], s["y"], gate=s["gate"], post=kind.get(c["post"], c["post"]), post_gain=s["post_gain"],
                               residual_scale=c["r"], pre=c["pre"], pre_gain=s["pre_gain"], scale=s["scale"], shift=s["shift"],
                               eps=EPS, dtype=dt)
    else:
        h, out = _norms(s["h"].float(), s["y"].float(), s["gate"], s["post_gain"], s["pre_gain"], s["scale"], s["shift"], c)
        h = h.to(s["h"].dtype)
        if dt == F8:
            codes, scale = _to_codes(out.flatten(0, 1), 1)
            out = codes.view(out.shape), scale.view(out.shape[0], out.shape[1], -1)
        else:
            out = out.to(dt)
    return {"h": h, "codes": out[0], "scale": out[1]} if dt == F8 else {"h": h, "out": out}


# ----------------------------------------------------------------- 64-bit results

def _tops(v):
    """Scales of the blocks of rows v in 64 bits."""
    return torch.stack([b.abs().amax(-1) for b in v.split(BLOCK, -1)], -1) / TOP


def _product(a, sa, b, sb):
    """Block by block: the sum of the codes' products times both scales."""
    out = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.float64, device="cuda")
    of = torch.arange(b.shape[0], device="cuda") // BLOCK
    for k, (x, w) in enumerate(zip(a.double().split(BLOCK, 1), b.double().split(BLOCK, 1))):
        out += (x @ w.t()) * sa[:, k, None].double() * sb[of, k].double()
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "quantize":
        x = s["x"].double()
        return {"codes": None, "scale": torch.stack([_tops(b.abs().amax(0)) for b in x.split(c["block"], 0)]) if c["block"] > 1 else _tops(x)}
    if c["kind"] == "matmul":
        out = _product(s["a"], s["a_scale"], s["b"], s["b_scale"])
        return out if s["bias"] is None else out + s["bias"].double()
    if c["kind"] == "gated":
        g, u = (_product(s["a"], s["a_scale"], s[n], s[n + "_scale"]) + (s[n + "_bias"].double() if c["bias"] else 0.0) for n in ("gate", "up"))
        if c["act"] == "silu":
            out = g * torch.sigmoid(g) * u
        else:
            out = g * torch.sigmoid(math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)) * u
        return {"codes": None, "scale": _tops(out)} if c["dtype"] == "f8" else out

    def norm(v, kind, gain):
        if kind == "none":
            return v
        v = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        v = v / (v.square().sum(-1, keepdim=True) / c["D"] + EPS).sqrt()
        return v if gain is None else v * gain.double()

    def each(v, n, other):
        if v is None:
            return other
        return v.double()[n] if v.dim() == 2 else v.double()

    hs, outs = [], []
    for n in range(c["S"]):
        h = s["h"][n].double() * c["r"] + each(s["gate"], n, 1.0) * norm(s["y"][n].double(), c["post"], s["post_gain"])
        hs.append(h)
        outs.append(norm(h, c["pre"], s["pre_gain"]) * (1.0 + each(s["scale"], n, 0.0)) + each(s["shift"], n, 0.0))
    h, out = torch.stack(hs), torch.stack(outs)
    return {"h": h, "codes": None, "scale": _tops(out)} if c["dtype"] == "f8" else {"h": h, "out": out}
