"""The sums behind products of e4m3 codes as a whole, in every kernel: those of bf16 outputs against the plain form of what the
8-bit instruction cuts off, those of fp32 outputs and of codes against exact ones."""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
import f8_sums as S  # noqa: E402
from f8_util import BF16, F8, FP32, U, blocks  # noqa: E402

ids = lambda v: str(v).replace("torch.", "")  # noqa: E731

# Rows, outputs and K (gated: 1152) that take every tile of their kind, and products in two launches.
PRODUCTS = [(8, 1152, 1152), (16, 520, 1152), (30, 1152, 1152), (100, 1152, 1152), (257, 2304, 1152), (520, 2304, 1152), (1100, 4200, 1601),
            (2060, 2304, 1152), (2100, 4200, 1152), (6000, 6000, 1152), (4160, 4200, 1152)]
GATED = [(8, 700), (30, 520), (100, 1152), (257, 2050), (100, 2304), (1100, 1152), (2060, 2304), (3000, 6000), (4150, 2050), (6000, 2050)]


@pytest.mark.parametrize("dtype", [BF16, FP32], ids=ids)
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_sums_of_products(M, N, K, dtype):
    """Equal rows, and a bias that is the result's opposite: what is left are the errors of the sums, which bf16 holds as well
    as fp32 does."""
    from paper_2511_22009_amd import matmul_f8
    (a, sa, b, sb), _ = S.operands(M, N, K, M + N, same_rows=True)
    want = S.exact_product(a[:1], sa[:1], b, sb)
    bias = (-want[0]).float()
    out = matmul_f8(a, sa, b, sb, bias, dtype=dtype).double()
    off = S.cut_product(a[:1], sa[:1], b, sb) - want if dtype == BF16 else torch.zeros_like(want)
    left = out - (off + want + bias.double())
    allowed = float(want.norm()) * S.step(K) + float(off.norm()) * 2.0 ** -8
    assert float(left.norm(dim=1).max()) <= allowed


@pytest.mark.parametrize("M,N", [(8, 512), (100, 512), (300, 2304)])
def test_bf16_outputs_are_their_sums_rounded(M, N):
    """But for those whose sum's own error reaches a tie: of a value that far off, the share of a step that it is."""
    from paper_2511_22009_amd import matmul_f8
    K = 1152
    args, _ = S.operands(M, N, K, M + N)
    out = matmul_f8(*args).double()
    exact = S.exact_product(*args)
    for sums, err in ((S.cut_product(*args), S.step(K) * exact.square().mean().sqrt()), (exact, (S.cut_product(*args) - exact).abs())):
        want = sums.to(BF16).double()
        bf16_step = torch.ldexp(torch.ones_like(want), S.power(sums) - 7)
        share = float(((err + S.step(K) * exact.square().mean().sqrt()) / bf16_step).clamp_max(1.0).mean())
        assert float((out != want).double().mean()) <= share + 6 * (share / out.numel()) ** 0.5
        if sums is not exact:
            assert bool(((out - want).abs() <= bf16_step + 2 * err).all())


@pytest.mark.parametrize("name", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,N", GATED)
def test_sums_of_gated_products(M, N, name):
    """fp32 values, and codes' scales, as exact as fp32 sums leave them: the 8-bit instruction's would be over five times further
    off than what is allowed."""
    from paper_2511_22009_amd import gated_matmul_f8
    args = S.gated_operands(M, N, 1152, M + N)
    want, err = S.gated(*args, name)
    assert S.whole(gated_matmul_f8(*args, activation=name, dtype=FP32), want, err) <= 1.0
    scale, scale_err = S.top_errors(want, err)
    assert S.whole(gated_matmul_f8(*args, activation=name, dtype=F8)[1], scale, scale_err) <= 1.0


@pytest.mark.parametrize("name", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,N", [(8, 700), (100, 520), (257, 520)])
def test_gated_bf16_outputs_are_their_sums_rounded(M, N, name):
    from paper_2511_22009_amd import gated_matmul_f8
    args = S.gated_operands(M, N, 1152, M + N)
    out = gated_matmul_f8(*args, activation=name, dtype=BF16).double()
    sums, err = S.gated(*args, name, product=S.cut_product)
    bf16_step = torch.ldexp(torch.ones_like(sums), S.power(sums) - 7)
    share = float((err / bf16_step).clamp_max(1.0).mean())
    assert float((out != sums.to(BF16).double()).double().mean()) <= share + 6 * (share / out.numel()) ** 0.5


@pytest.mark.parametrize("name", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K", [(1100, 1152, 1152), (520, 2304, 1152), (1300, 1500, 700), (1100, 2500, 260)])
def test_codes_are_those_of_the_values(M, N, K, name):
    """Where the fp32 call adds blocks in the order of codes, in a whole tile: the bits that quantize_f8 gives of its values."""
    from paper_2511_22009_amd import gated_matmul_f8, quantize_f8
    args = S.gated_operands(M, N, K, M + N)
    q, s = gated_matmul_f8(*args, activation=name, dtype=F8)
    want, scale = quantize_f8(gated_matmul_f8(*args, activation=name, dtype=FP32))
    assert torch.equal(s, scale) and torch.equal(q.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("M,N", GATED)
def test_codes_are_nearly_those_of_the_values(M, N):
    """In another order, but for values that are a rounding of the sums from a tie: the share of a code's step that it is. Both
    sides have such an error, and that of the scale."""
    from paper_2511_22009_amd import gated_matmul_f8, quantize_f8
    args = S.gated_operands(M, N, 1152, M + N)
    q, s = gated_matmul_f8(*args, dtype=F8)
    want, scale = quantize_f8(gated_matmul_f8(*args, dtype=FP32))
    exact, err = S.gated(*args, "silu")
    top, top_err = S.top_errors(exact, err)
    assert float((s.double() - scale.double()).norm()) <= 2 * float(top_err.norm())
    of = lambda t: t.repeat_interleave(128, 1)[:, :N]  # noqa: E731
    code = exact.abs() / of(top)
    code_step = torch.ldexp(torch.ones_like(code), S.power(code).clamp_min(-6) - 3)
    share = float((2 * (err / of(top) + code * of(top_err / top)) / code_step).clamp_max(1.0).mean())
    differ = q.view(torch.uint8) != want.view(torch.uint8)
    assert float(differ.double().mean()) <= share + 6 * (share / differ.numel()) ** 0.5
    # neighbours: the order of codes is that of their bits; a sign that differs is that of a value next to 0
    assert bool(((q.float().abs() - want.float().abs()).abs() <= 1.01 * code_step + U).all())
    assert s.shape == (M, blocks(N))
