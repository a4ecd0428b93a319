"""A model whose block projections run in 8 bits (sf_set_int8), stage by stage against 64-bit
arithmetic on the same codes.

What a stage reads is taken from the model itself (residual stream, adaLN table, attention and
MLP buffers), so its codes are known: exactly where it reads bf16, and up to a few codes next to
a half where LayerNorm's fp32 values lie within their rounding of one.
"""
import os
from dataclasses import replace

import numpy as np
import pytest

import oracle
import workloads as W
from conftest import blob_for
from helpers import bf16_round, rel_l2_per_sample

pytestmark = pytest.mark.gpu

from gpu_util import dev, host, torch  # noqa: E402

U = 2.0 ** -24
BF = 2.0 ** -8

# width 88 and MLP width 360 are no multiples of 16: rows of codes end inside a 16-byte piece
ODD = replace(W.get_config("tiny_tsens"), name="odd88", D=88, heads=1, mlp=360, H=12, W=20, K=3, schedule="uniform3")
CASES = {n: W.get_config(n) for n in ("tiny_tsens", "ragged", "dh72", "short16", "tiny_cfg")}
CASES["odd88"] = ODD


def blob_of(name):
    return W.make_blob(ODD) if name == "odd88" else blob_for(name)


def load(name, rows=8, prec="bf16"):
    from paper_2511_22009_amd import Model, Precision
    return Model(blob_of(name), Precision[prec.upper()], rows)


def codes64(x):
    """Codes and scales (fp32 values) of the rows of x, in fp64."""
    a = x.abs().amax(1)
    q = torch.round(127.0 * x / torch.where(a > 0, a, torch.ones_like(a))[:, None])
    return q, (a.float() / 127.0).double()


def weights64(w):
    return codes64(dev(bf16_round(w)).double())


def ln_mod(h, shift, scale):
    d = h - h.mean(-1, keepdim=True)
    return d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-6) * (1.0 + scale) + shift


def gelu(u):
    return 0.5 * u * (1.0 + torch.tanh(np.sqrt(2.0 / np.pi) * (u + 0.044715 * u ** 3)))


def product(x, w):
    """The product of codes, and what one code more or less could change it by."""
    (qx, sx), (qw, sw) = codes64(x), w
    return (qx @ qw.t()) * sx[:, None] * sw, sx[:, None] * sw * 127.0


def off(got, want, allowed):
    assert torch.isfinite(got.double()).all()
    return float(((got.double() - want).abs() / (allowed + 1e-30)).max())


def conditioning(cfg):
    from paper_2511_22009_amd import Cond
    if not cfg.has_cross:
        return None
    return Cond(dev(W.context(cfg, cfg.K)), dev(W.null_context(cfg)), cfg.guidance)


@pytest.mark.parametrize("name", [n for n in CASES if n != "tiny_cfg"])
def test_every_projection_of_every_block(name):
    """A code next to a half may fall either way; more than FEW of a row's do not (they lie within
    16 U of a half with a chance of 16 U x 127 x 2, some 2e-4, each)."""
    from paper_2511_22009_amd import Buffer
    FEW = 3
    cfg = CASES[name]
    om = oracle.load_blob(blob_of(name))
    m = load(name)
    m.set_int8()
    t, _ = W.slot_times(cfg)
    x = dev(W.latents(cfg, cfg.K))
    K, N, D, H = cfg.K, cfg.N, cfg.D, cfg.heads
    table = m.modulation(t).double()
    for l in range(cfg.L):
        h = m.residual(x, t, l).double()
        out = m.residual(x, t, l + 1).double()
        mod = [table[:, l * 6 * D + i * D:l * 6 * D + (i + 1) * D].repeat_interleave(N, 0) for i in range(6)]
        h = h.reshape(K * N, D)
        b = {k: om.blocks[l][k] for k in om.blocks[l]}
        bias = {k: dev(b[k]).double() for k in ("b_qkv", "b_o", "b_fc1", "b_fc2")}
        # QKV, heads apart
        p, one = product(ln_mod(h, mod[0], mod[1]), weights64(b["W_qkv"]))
        want = p + bias["b_qkv"]
        allowed = BF * want.abs() + 24 * U * (p.abs() + want.abs()) + FEW * one
        parts = lambda z: z.reshape(K, N, 3, H, cfg.dh).permute(2, 0, 3, 1, 4)  # noqa: E731
        w3, a3 = parts(want), parts(allowed)
        shape = (K, H, N, cfg.dh)
        assert off(m.debug_read(Buffer.Q, shape), w3[0], a3[0]) <= 1.0
        assert off(m.debug_read(Buffer.K, shape), w3[1], a3[1]) <= 1.0
        ld = m.info["vt_ld"]
        col = torch.arange(N, device="cuda")
        col = (col & ~12) | ((col & 4) << 1) | ((col & 8) >> 1)
        vt = m.debug_read(Buffer.VT, (K, H, cfg.dh, ld))
        assert off(vt[..., col].transpose(2, 3), w3[2], a3[2]) <= 1.0
        rest = torch.ones(ld, dtype=torch.bool, device="cuda")
        rest[col] = False
        assert not vt[..., rest].any()                       # columns of no key stay zero
        # attention output: codes of bf16 rows are exact
        o = m.debug_read(Buffer.ATTN, (K * N, D)).double()
        p1, _ = product(o, weights64(b["W_o"]))
        y1 = p1 + bias["b_o"]
        h1 = h + mod[2] * y1
        # MLP up
        p, one = product(ln_mod(h1, mod[3], mod[4]), weights64(b["W_fc1"]))
        u = p + bias["b_fc1"]
        f = m.debug_read(Buffer.MLP, (K * N, cfg.mlp))
        want = gelu(u)                                        # its slope is at most 1.13
        allowed = BF * want.abs() + 32 * U * (p.abs() + u.abs()) + 1.13 * FEW * one
        assert off(f, want, allowed) <= 1.0
        # MLP down
        p2, _ = product(f.double(), weights64(b["W_fc2"]))
        y2 = p2 + bias["b_fc2"]
        want = h1 + mod[5] * y2
        allowed = 8 * U * (h.abs() + (mod[2] * y1).abs() + (mod[2] * p1).abs() + (mod[5] * y2).abs() + (mod[5] * p2).abs() + want.abs())
        assert off(out.reshape(K * N, D), want, allowed) <= 1.0
    m.close()


@pytest.mark.parametrize("name", ["tiny_tsens", "ragged", "tiny_cfg"])
def test_velocity_is_near_the_oracle(name):
    """A rounding to 127 steps of a row's largest magnitude (at most 4.5 of its rms) is off by 4.5 /
    127 / sqrt 12 = 1.0 % rms, two factors 1.5 % of a projection's output, four projections in a
    block 3 %; guidance multiplies the difference of two rows' errors by 7.5."""
    from paper_2511_22009_amd import Cond
    cfg = CASES[name]
    om = oracle.load_blob(blob_of(name))
    m = load(name)
    t, _ = W.slot_times(cfg)
    x = W.latents(cfg, cfg.K)
    cond = conditioning(cfg)
    plain = host(m.velocity(dev(x), t, cond))
    m.set_int8()
    got = host(m.velocity(dev(x), t, cond))
    if cond is None:
        want = oracle.velocity(om, x, t)
    else:
        want = oracle.velocity(om, x, t, W.context(cfg, cfg.K), W.null_context(cfg), cfg.guidance)
    assert max(rel_l2_per_sample(got, want)) <= (0.03 if cond is None else 0.03 * 7.5)
    assert not np.array_equal(got, plain)
    np.testing.assert_array_equal(host(m.velocity(dev(x), t, cond)), got)       # the same bits again
    m.set_int8(False)
    np.testing.assert_array_equal(host(m.velocity(dev(x), t, cond)), plain)
    m.close()
    if cond is not None:
        assert isinstance(cond, Cond)


@pytest.mark.parametrize("name", ["ragged", "odd88"])
def test_rows_do_not_depend_on_the_batch(name):
    cfg = CASES[name]
    m = load(name)
    m.set_int8()
    t, _ = W.slot_times(cfg)
    x = dev(W.latents(cfg, cfg.K))
    whole = m.velocity(x, t)
    for k in range(cfg.K):
        assert torch.equal(whole[k:k + 1], m.velocity(x[k:k + 1].contiguous(), t[k:k + 1]))
    m.close()


def test_together_with_turned_queries_and_keys_in_replayed_steps():
    from paper_2511_22009_amd import Rotary
    cfg = CASES["tiny_tsens"]
    t, dt = W.slot_times(cfg)
    x0 = W.latents(cfg, cfg.K)
    z = dev(W.z_new_for_image(cfg, 2))
    m = load("tiny_tsens")
    s = torch.cuda.Stream()
    seen = []
    for on in (True, False, True):
        m.set_int8(on)
        m.set_qk(rotary=Rotary([16, 16], layout="halves"))
        m.graph_enable(False)
        eager, done = dev(x0), torch.empty(cfg.latent_shape, device="cuda")
        m.stream_step(eager, t, dt, cfg.K, z, done, stream=s)
        s.synchronize()
        m.graph_enable(True)
        for _ in range(3):
            x, d = dev(x0), torch.empty(cfg.latent_shape, device="cuda")
            torch.cuda.synchronize()
            m.stream_step(x, t, dt, cfg.K, z, d, stream=s)
            s.synchronize()
            assert torch.equal(x, eager) and torch.equal(d, done)
            torch.randn(1 << 16, device="cuda").sum().item()
        seen.append(eager)
    assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])
    m.close()


def test_refusals_and_failed_allocation(monkeypatch):
    from paper_2511_22009_amd import SFError
    m = load("tiny_tsens", prec="fp32")
    with pytest.raises(SFError) as e:
        m.set_int8()
    assert e.value.code == -1
    m.set_int8(False)
    m.close()
    cfg = CASES["tiny_tsens"]
    m = load("tiny_tsens")
    t, _ = W.slot_times(cfg)
    x = dev(W.latents(cfg, cfg.K))
    plain = m.velocity(x, t)
    monkeypatch.setenv("SF_FAIL_ALLOC_AFTER", "0")
    with pytest.raises(SFError) as e:
        m.set_int8()
    assert e.value.code == -4
    os.environ.pop("SF_FAIL_ALLOC_AFTER")
    assert torch.equal(m.velocity(x, t), plain)
    m.set_int8()
    assert not torch.equal(m.velocity(x, t), plain)
    m.close()


def test_many_rows():
    """64 rows in one call: every row as alone."""
    cfg = CASES["ragged"]
    m = load("ragged", rows=64)
    m.set_int8()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((64,) + cfg.latent_shape, generator=g, device="cuda")
    t = np.linspace(1.0, 0.02, 64).astype(np.float32)
    whole = m.velocity(x, t)
    for k in (0, 17, 63):
        assert torch.equal(whole[k:k + 1], m.velocity(x[k:k + 1].contiguous(), t[k:k + 1]))
    m.close()
