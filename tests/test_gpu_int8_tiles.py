"""8-bit projections at the sizes where every tile of every epilogue runs, and for rows under
guidance with cross-attention between the 8-bit stages.

Stage by stage against 64-bit arithmetic on the same codes, as in test_gpu_int8.py, whose tolerances
hold here: a code of a LayerNorm's row may fall either way next to a half, with a chance of some
2e-4 each, so a row of up to 1152 has 0.3 of them on average and more than FEW hardly ever, and those
of chance signs; the rest counts roundings.
"""
from dataclasses import replace

import numpy as np
import pytest

import oracle
import workloads as W
from helpers import bf16_round

pytestmark = pytest.mark.gpu

from gpu_util import dev, torch  # noqa: E402
from test_gpu_int8 import BF, U, gelu, ln_mod, off, product, weights64  # noqa: E402

FEW = 3


def net(D, heads, mlp, gh, gw, **kw):
    return W.Config("net", C=4, H=2 * gh, W=2 * gw, p=2, D=D, L=1, heads=heads, mlp=mlp, init="tsens", **kw)


# one block each: the networks' widths at 512^2 with four slots, and sizes that end inside a tile
# and take the other tiles (test_operators_edges_cpu.py asserts that each runs): (network, rows)
SHAPES = [(net(768, 12, W.get_config("s512").mlp, 32, 32), 4), (net(1152, 16, 4608, 32, 32), 4), (net(1152, 16, 4608, 31, 29), 3),
          (net(64, 1, 136, 8, 9), 1), (net(88, 1, 272, 32, 33), 8), (net(512, 4, 1032, 8, 9), 1), (net(384, 6, 1160, 32, 33), 8),
          (net(192, 4, 584, 28, 33), 8), (net(1024, 8, 3080, 14, 23), 2), (net(512, 4, 1032, 32, 33), 8), (net(640, 8, 1288, 32, 33), 8),
          (net(1024, 8, 2056, 32, 33), 8)]
name_of = lambda s: f"{s[0].D}x{s[0].mlp}x{s[0].N}x{s[1]}"  # noqa: E731


def load(blob, rows):
    from paper_2511_22009_amd import Model, Precision
    m = Model(blob, Precision.BF16, rows)
    m.set_int8()
    return m


def times(n):
    return np.linspace(1.0, 0.05, n).astype(np.float32)


def inputs(cfg, n):
    g = torch.Generator(device="cuda").manual_seed(cfg.D + cfg.N + n)
    return torch.randn((n,) + cfg.latent_shape, generator=g, device="cuda"), times(n)


def modulation(m, cfg, t, rows):
    """The block's six vectors for every token row; row r takes the table's slot r modulo the slots."""
    table = m.modulation(t).double()
    slot = torch.arange(rows, device="cuda") % len(t)
    D = cfg.D
    return [table[slot, i * D:(i + 1) * D].repeat_interleave(cfg.N, 0) for i in range(6)]


def heads_apart(z, cfg, rows):
    return z.reshape(rows, cfg.N, -1, cfg.heads, cfg.dh).permute(2, 0, 3, 1, 4)


def check_qkv(m, cfg, h, mod, b, rows, queries=True):
    from paper_2511_22009_amd import Buffer
    p, one = product(ln_mod(h, mod[0], mod[1]), weights64(b["W_qkv"]))
    want = p + dev(b["b_qkv"]).double()
    allowed = BF * want.abs() + 24 * U * (p.abs() + want.abs()) + FEW * one
    w3, a3 = heads_apart(want, cfg, rows), heads_apart(allowed, cfg, rows)
    shape = (rows, cfg.heads, cfg.N, cfg.dh)
    if queries:
        assert off(m.debug_read(Buffer.Q, shape), w3[0], a3[0]) <= 1.0
    assert off(m.debug_read(Buffer.K, shape), w3[1], a3[1]) <= 1.0
    ld = m.info["vt_ld"]
    col = torch.arange(cfg.N, device="cuda")
    col = (col & ~12) | ((col & 4) << 1) | ((col & 8) >> 1)
    vt = m.debug_read(Buffer.VT, (rows, cfg.heads, cfg.dh, ld))
    assert off(vt[..., col].transpose(2, 3), w3[2], a3[2]) <= 1.0
    rest = torch.ones(ld, dtype=torch.bool, device="cuda")
    rest[col] = False
    assert not vt[..., rest].any()


def after_attention(cfg, h, o, mod, b):
    """The residual rows past the attention's output projection, and the sizes that their roundings go by."""
    p, _ = product(o, weights64(b["W_o"]))
    y = p + dev(b["b_o"]).double()
    return h + mod[2] * y, h.abs() + (mod[2] * y).abs() + (mod[2] * p).abs()


def check_mlp(m, cfg, h1, size, mod, b, out, rows):
    from paper_2511_22009_amd import Buffer
    p, one = product(ln_mod(h1, mod[3], mod[4]), weights64(b["W_fc1"]))
    u = p + dev(b["b_fc1"]).double()
    f = m.debug_read(Buffer.MLP, (rows * cfg.N, cfg.mlp))
    want = gelu(u)                                            # its slope is at most 1.13
    assert off(f, want, BF * want.abs() + 32 * U * (p.abs() + u.abs()) + 1.13 * FEW * one) <= 1.0
    p2, _ = product(f.double(), weights64(b["W_fc2"]))
    y = p2 + dev(b["b_fc2"]).double()
    want = h1 + mod[5] * y
    assert off(out, want, 8 * U * (size + (mod[5] * y).abs() + (mod[5] * p2).abs() + want.abs())) <= 1.0


@pytest.mark.parametrize("cfg,rows", SHAPES, ids=map(name_of, SHAPES))
def test_every_projection_in_every_tile(cfg, rows):
    from paper_2511_22009_amd import Buffer
    blob = W.make_blob(cfg)
    b = oracle.load_blob(blob).blocks[0]
    m = load(blob, rows)
    x, t = inputs(cfg, rows)
    flat = (rows * cfg.N, cfg.D)
    h = m.residual(x, t, 0).double().reshape(flat)
    out = m.residual(x, t, 1)
    mod = modulation(m, cfg, t, rows)
    check_qkv(m, cfg, h, mod, b, rows)
    h1, size = after_attention(cfg, h, m.debug_read(Buffer.ATTN, flat).double(), mod, b)
    check_mlp(m, cfg, h1, size, mod, b, out.reshape(flat), rows)
    # a row alone takes other tiles, and has the same bits
    for k in {0, rows - 1}:
        assert torch.equal(m.residual(x[k:k + 1].contiguous(), t[k:k + 1], 1), out[k:k + 1])
    m.close()


def test_guided_rows_with_cross_attention():
    """Conditional and unconditional rows share their slot's modulation and, in the first block, all
    of the self-attention: its keys and values in both halves are those of the same network without
    cross-attention, bit for bit, whose queries and attention output are read there. What the
    cross-attention adds is computed from its own output."""
    from paper_2511_22009_amd import Buffer, Cond
    cfg = net(128, 4, 520, 10, 14, ctx_len=20, ctx_dim=64, has_cross=1, cfg=True)
    K, rows = 3, 6
    tensors = W.make_weights(cfg)
    plain_cfg = replace(cfg, has_cross=0, ctx_len=0, ctx_dim=0)
    blob = W.make_blob(cfg, tensors=tensors)
    b = oracle.load_blob(blob).blocks[0]
    m, plain = load(blob, rows), load(W.make_blob(plain_cfg, tensors=tensors), rows)
    x, t = inputs(cfg, K)
    cond = Cond(dev(W.context(cfg, K)), dev(W.null_context(cfg)), 7.5)
    h = m.residual(x, t, 0, cond).double()
    assert torch.equal(h[:K], h[K:])
    h = h.reshape(rows * cfg.N, cfg.D)
    out = m.residual(x, t, 1, cond)
    mod = modulation(m, cfg, t, rows)
    check_qkv(m, cfg, h, mod, b, rows, queries=False)
    plain.residual(x, t, 1)
    ld = m.info["vt_ld"]
    for buffer, shape in ((Buffer.K, (cfg.heads, cfg.N, cfg.dh)), (Buffer.VT, (cfg.heads, cfg.dh, ld))):
        both, alone = m.debug_read(buffer, (rows,) + shape), plain.debug_read(buffer, (K,) + shape)
        assert torch.equal(both[:K], alone) and torch.equal(both[K:], alone)
    check_qkv(plain, plain_cfg, h[:K * cfg.N], [v[:K * cfg.N] for v in mod], b, K)
    o = plain.debug_read(Buffer.ATTN, (K * cfg.N, cfg.D)).double().repeat(2, 1)
    h1, size = after_attention(cfg, h, o, mod, b)
    # cross-attention's output projection: bf16 weights, a sum of D products and the bias in fp32
    ox = m.debug_read(Buffer.ATTN, (rows * cfg.N, cfg.D)).double()
    w = dev(bf16_round(b["W_ox"])).double()
    y = ox @ w.t() + dev(b["b_ox"]).double()
    h2 = h1 + y
    size = size + y.abs() + (cfg.D / 8) * (ox.abs() @ w.abs().t())      # D roundings, in the eights of check_mlp
    check_mlp(m, cfg, h2, size, mod, b, out.reshape(rows * cfg.N, cfg.D), rows)
    m.close()
    plain.close()


@pytest.mark.parametrize("name", ["tiny_cfg", "tiny_cfg_ctx20"])
def test_guided_velocity_is_its_two_halves(name):
    """Guidance in 8 bits: v = v_u + w (v_c - v_u) of runs without guidance, with the slots' contexts
    and with the null context in their place, within the roundings of that formula."""
    from conftest import blob_for
    from paper_2511_22009_amd import Cond
    cfg = W.get_config(name)
    m = load(blob_for(name), 8)
    x, t = inputs(cfg, cfg.K)
    ctx, null, w = dev(W.context(cfg, cfg.K)), dev(W.null_context(cfg)), 7.5
    v = m.velocity(x, t, Cond(ctx, null, w)).double()
    c = m.velocity(x, t, Cond(ctx)).double()
    u = m.velocity(x, t, Cond(null[None].repeat(cfg.K, 1, 1).contiguous())).double()
    want = u + w * (c - u)
    allowed = U * ((c - u).abs() * 2 * w + want.abs())            # difference, product, sum
    assert off(v, want, allowed) <= 1.0
    assert float((c - u).abs().max()) > 0
    m.close()
