"""The operators in 8-bit floating point and the norms around a block where their ranges end."""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
import f8_util as P  # noqa: E402
from f8_util import BF16, F8, FP32, U, gen, randn, worst  # noqa: E402

ids = lambda v: str(v).replace("torch.", "")  # noqa: E731


def add_one_in_place(rows, shape):
    """h' = h + 1 over h itself, and nothing behind it."""
    from paper_2511_22009_amd import residual_norm
    room = torch.zeros(rows + (1 << 22), device="cuda", dtype=BF16)
    h = room[:rows].view(shape)
    y = torch.ones((1, 1, 1), device="cuda", dtype=BF16).expand(shape)
    out, none = residual_norm(h, y, h_out=h)
    assert out is h and none is None
    for part in room[:rows].split(1 << 28):
        assert bool((part == 1).all())
    assert not room[rows:].any()


def test_residual_norm_of_as_many_samples_as_it_takes():
    """1024 launches; the first sample past the last one is 2^31."""
    rows = (1 << 31) - 1
    add_one_in_place(rows, (rows, 1, 1))


def test_residual_norm_of_as_many_tokens_as_it_takes():
    """One sample, its last workgroup's rows up to the last; the first row past them is 2^31."""
    rows = (1 << 31) - 1
    add_one_in_place(rows, (1, rows, 1))


def constant_rows(D, dtype, eps=1e-6):
    """Rows of one value each, of every size, and their norms after and before a block."""
    from paper_2511_22009_amd import residual_norm
    sizes = torch.tensor([0.0, 1e-40, 1e-30, 1e-10, 1.0, 1000.1, 1e10, 1e15, 1.1e19, 1e20, 7e24, 1e30, 3e38], device="cuda")
    h = torch.cat([sizes, -sizes])[:, None].expand(-1, D).contiguous()
    none = torch.zeros_like(h)
    shift = torch.linspace(-2, 3, D, device="cuda")
    gate = torch.full((D,), 0.5, device="cuda")
    for n in (1, 300):  # few rows and many are different kernels
        x, y = h.repeat(n, 1), none.repeat(n, 1)
        out = residual_norm(x, y, pre="layer", shift=shift, dtype=FP32, eps=eps)[1]
        assert torch.equal(out, shift.expand_as(x))
        after = residual_norm(y, x, post="layer", gate=gate, dtype=FP32, eps=eps)[0]
        assert not after.any()
        for kind in ("rms", "layer"):
            q = residual_norm(x, y, pre=kind, dtype=dtype, eps=eps)[1]
            q, s = q if dtype == F8 else (q, q)
            assert torch.isfinite(q.float()).all() and torch.isfinite(s.float()).all()
            assert kind == "rms" or not (q.float().any() or s.any())


@pytest.mark.parametrize("eps", [1e-6, 1e-30])
@pytest.mark.parametrize("dtype", [BF16, FP32, F8], ids=ids)
@pytest.mark.parametrize("D", [1, 2, 64, 128, 512, 2048, 4096])
def test_layer_norm_of_constant_rows(D, dtype, eps):
    """No deviation and an eps above 0: the norm is 0, whatever the size. Sums of powers of two of one value are exact."""
    constant_rows(D, dtype, eps)


@pytest.mark.parametrize("eps", [1e-6, 1e-30])
@pytest.mark.parametrize("dtype", [BF16, FP32, F8], ids=ids)
@pytest.mark.parametrize("D", [3, 5, 100, 129, 257, 770, 771, 1000, 1152, 1276, 1800, 3000, 5000, 8191, 16384])
def test_layer_norm_of_constant_rows_whose_mean_is_rounded(D, dtype, eps):
    """A mean that is some steps off leaves a deviation of that in every value, and their mean takes it off."""
    constant_rows(D, dtype, eps)


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("D", [2, 5, 128, 257, 770, 1000, 1152, 2044, 5000, 16384])
def test_layer_norm_of_rows_of_nearly_one_value(D, eps):
    """Values a few steps of fp32 apart: their deviations are whole steps, which the mean's rounding must not hide.

    What the first mean leaves are whole steps, exactly; of these the mean is off by U of it, each deviation by U of itself, and
    so is what their own mean takes off: under 4 U of the row's largest deviation. The root of the mean square has as many
    roundings of a partial sum as in f8_util.norm, and six more."""
    from paper_2511_22009_amd import residual_norm
    g = gen(D)
    for n in (1, 200):
        base = torch.tensor([1e-30, 1e-10, 1.0, 1000.1, 1e10, 1e15, 1e20, 1e30, 3e38], device="cuda") * (1 - 0.3 * torch.rand(9, generator=g, device="cuda"))
        base = torch.cat([base, -base])
        steps = torch.randint(-3, 4, (18, D), generator=g, device="cuda", dtype=torch.int32)
        steps[::3] *= torch.rand((6, D), generator=g, device="cuda") < 0.1
        steps[1::3] = 0
        steps[:, 0] = 1                                    # at least one value is another
        steps[:, -1] = 0
        x = (base.view(torch.int32)[:, None] + steps).view(FP32)
        off = x.double() - base.double()[:, None]
        off = off - off.mean(-1, keepdim=True)
        want = off / (off.square().mean(-1, keepdim=True) + eps).sqrt()
        allowed = (want.abs() + want.abs().amax(-1, keepdim=True)) * (D / 64 + 12 + 10) * U
        x, y = x.repeat(n, 1), torch.zeros((18 * n, D), device="cuda")
        pre = residual_norm(x, y, pre="layer", dtype=FP32, eps=eps)[1]
        post = residual_norm(y, x, post="layer", eps=eps)[0]
        assert worst(pre, want.repeat(n, 1), allowed.repeat(n, 1)) <= 1.0
        assert worst(post, want.repeat(n, 1), allowed.repeat(n, 1)) <= 1.0


def test_layer_norm_next_to_the_largest_number():
    """Rows whose values lose fp32's range when their mean is taken off, but for a scale."""
    from paper_2511_22009_amd import residual_norm
    top = torch.finfo(FP32).max
    x = torch.tensor([[top, -top * (1 - 2.0 ** -5)], [top, -top], [top, 0.0], [-top, -top * (1 - 2.0 ** -20)]], device="cuda")
    for D in (2, 1152):
        h = x.repeat(1, D // 2)
        out = residual_norm(h, torch.zeros_like(h), pre="layer", dtype=FP32)[1]
        assert worst(out, torch.tensor([1.0, -1.0], device="cuda", dtype=torch.float64).repeat(4, D // 2) * torch.tensor([[1], [1], [1], [-1.0]], device="cuda"),
                     torch.full((4, D), (D / 64 + 32) * U, device="cuda", dtype=torch.float64)) <= 1.0


def given_results():
    """(results that are given, call that writes them) for every operator."""
    from paper_2511_22009_amd import (Rotary, gated_matmul_f8, matmul_f8, matmul_i8, qk_norm_rotate, quantize_f8, quantize_rows,
                                      residual_norm, rotate)
    g = gen(11)
    x, h, pos, y = randn(g, 40, 64), randn(g, 2, 5, 3, 64), randn(g, 5, 2), randn(g, 40, 64)
    r, f8 = Rotary([32, 32]), lambda t: torch.zeros_like(t).to(F8)
    i8, si8 = quantize_rows(x)
    a, sa = quantize_f8(x)
    w, sw = quantize_f8(x, 128)
    e = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    for call, outs in (
            (lambda o, s: quantize_rows(x, o, s), (torch.zeros_like(i8), e(40))), (lambda o: matmul_i8(i8, si8, i8, si8, out=o), (e(40, 40),)),
            (lambda o: rotate(o, pos, r, out=o), (h.clone(),)),
            (lambda q, k: qk_norm_rotate(q, k, positions=pos, rotary=r, out=(q, k)), (h.clone(), h.clone())),
            (lambda o, s: quantize_f8(x, 1, o, s), (f8(x), e(40, 1))), (lambda o: matmul_f8(a, sa, w, sw, out=o), (e(40, 40),)),
            (lambda o, s: gated_matmul_f8(a, sa, w, sw, w, sw, out=o, out_scale=s), (f8(e(40, 48))[:, :40], e(40, 1))),
            (lambda o, n, s: residual_norm(o, y, pre="rms", h_out=o, out=n, out_scale=s), (x.clone(), f8(x), e(40, 1)))):
        yield outs, call


def test_results_that_are_given_count_as_changed():
    """A backward pass that kept the old values ends with an error, as after torch's own writes."""
    for outs, call in given_results():
        before = [t._version for t in outs]
        call(*outs)
        assert [t._version for t in outs] == [v + 1 for v in before]
    from paper_2511_22009_amd import residual_norm
    h = torch.ones((4, 64), device="cuda")
    w = torch.ones((4, 64), device="cuda", requires_grad=True)
    loss = (w * h).sum()
    residual_norm(h, h.clone(), h_out=h)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_results_that_are_given_in_inference_mode():
    with torch.inference_mode():
        for outs, call in given_results():
            call(*outs)
        room = torch.zeros((4, 64), device="cuda")
    from paper_2511_22009_amd import residual_norm
    with torch.no_grad():
        assert residual_norm(room, torch.ones((4, 64), device="cuda"), h_out=room)[0] is room and bool((room == 1).all())


def test_tensors_with_a_forward_mode_tangent_are_refused():
    import torch.autograd.forward_ad as fw
    from paper_2511_22009_amd import quantize_f8, quantize_rows, residual_norm
    x = randn(gen(12), 4, 64)
    for call in (quantize_rows, quantize_f8, lambda t: residual_norm(t, x, pre="rms"), lambda t: residual_norm(x, x, pre="rms", pre_gain=t[0])):
        want = call(x)
        with torch.no_grad(), fw.dual_level():
            d = fw.make_dual(x, torch.ones_like(x))
            with pytest.raises(TypeError, match="tangent"):
                call(d)
            got = call(fw.unpack_dual(d).primal)
        for p, q in zip(got, want):
            assert torch.equal(p.float(), q.float())


@pytest.mark.parametrize("N,K", [(1152, 1152), (300, 4400), (4200, 1601)])
def test_rows_do_not_see_each_other_but_for_the_order_of_sums(N, K):
    """Codes whose products are multiples of 2^-6 and scales of 1: every sum is below 14.1 K < 2^17 and a multiple of 2^-6, so exact
    in fp32 in every order. Then a row has the same bits in calls of every size, tile and number of launches."""
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8
    g = gen(N + K)
    M = 4160
    (a, sa), (w, sw), (u, su) = (P.codes(g, n, K, b) for n, b in ((M, 1), (N, 128), (N, 128)))
    for q in (a, w, u):
        P.narrow(q)
    sa, sw, su = sa.sign(), sw.sign(), su.sign()
    small = 2.0 ** -12
    for call in (lambda m: matmul_f8(a[m], sa[m], w, sw), lambda m: matmul_f8(a[m], sa[m], w, sw, dtype=FP32),
                 lambda m: gated_matmul_f8(a[m], sa[m], w, sw * small, u, su, dtype=BF16),
                 lambda m: gated_matmul_f8(a[m], sa[m], w, sw * small, u, su, dtype=FP32),
                 lambda m: gated_matmul_f8(a[m], sa[m], w, sw * small, u, su, dtype=F8)):
        whole = call(slice(0, M))
        for m in (slice(0, 1), slice(7, 23), slice(1, 33), slice(100, 165), slice(1000, 1300), slice(3000, 4100), slice(4100, M)):
            part = call(m)
            for p, q in zip(*((v if isinstance(v, tuple) else (v,)) for v in (part, whole))):
                p, q = (t.view(torch.uint8) if t.dtype == F8 else t for t in (p, q[m]))
                assert torch.equal(p, q)


def test_rows_that_become_codes_do_not_see_each_other():
    """Their blocks are added in one order in every tile and part: the same bits, whatever else is in the call."""
    from paper_2511_22009_amd import gated_matmul_f8
    for M, N, K in ((2100, 2048, 2301), (1300, 300, 1152)):
        g = gen(M)
        (a, sa), (w, sw), (u, su) = (P.codes(g, n, K, b) for n, b in ((M, 1), (N, 128), (N, 128)))
        call = lambda m: gated_matmul_f8(a[m], sa[m], w, sw, u, su, activation="gelu_tanh", dtype=F8)  # noqa: E731
        q, s = call(slice(0, M))
        for m in (slice(0, 1), slice(5, 38), slice(600, 900), slice(200, M - 1)):
            p, t = call(m)
            assert torch.equal(p.view(torch.uint8), q[m].view(torch.uint8)) and torch.equal(t, s[m])


def test_offsets_past_32_bits():
    """Tensors of over 2^32 entries: what lies on both sides of 2^31, 2^32 and at the end is what smaller calls give there."""
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, quantize_f8, residual_norm
    g = gen(70)
    M, W = 70001, 65536
    rows = [*range(5), *range(32766, 32770), *range(65534, 65538), *range(M - 5, M)]
    x = torch.zeros((M, W), device="cuda", dtype=BF16)
    x[rows] = randn(g, len(rows), W, dtype=BF16)
    a, sa = quantize_f8(x)
    want = quantize_f8(x[rows])
    assert torch.equal(a.view(torch.uint8)[rows], want[0].view(torch.uint8)) and torch.equal(sa[rows], want[1])
    assert int(torch.count_nonzero(sa.any(1))) == len(rows)
    # a product that reads them, and one that writes as many
    b, sb = P.codes(g, 40, W, 128)
    out = matmul_f8(a, sa, b, sb, dtype=FP32)
    P.check(out[rows], *P.product(a[rows], sa[rows], b, sb, exact=True), FP32)
    del x, a, sa, out
    (a, sa), (b, sb), (u, su) = (P.codes(g, n, 48, r) for n, r in ((M, 1), (W, 128), (W, 128)))
    out = matmul_f8(a, sa, b, sb)
    P.check(out[rows], *P.product(a[rows], sa[rows], b, sb, exact=False), BF16)
    del out
    q, s = gated_matmul_f8(a, sa, b, sb, u, su, dtype=F8)
    want = gated_matmul_f8(a[rows], sa[rows], b, sb, u, su, dtype=F8)   # codes have one order of sums
    assert torch.equal(q.view(torch.uint8)[rows], want[0].view(torch.uint8)) and torch.equal(s[rows], want[1])
    del q, s, a, b, u
    T, D = 131100, 16384
    tokens = [0, 1, *range(65534, 65538), T - 2, T - 1]
    h = torch.ones((2, T, D), device="cuda", dtype=BF16)
    part = randn(g, 2, len(tokens), D, dtype=BF16)
    h[:, tokens] = part
    y = randn(g, 1, 1, D, dtype=BF16)
    want, (wq, ws) = residual_norm(part, y.expand(2, len(tokens), -1).contiguous(), post="rms", pre="layer", dtype=F8)
    got, (q, s) = residual_norm(h, y.expand(2, T, -1), post="rms", pre="layer", dtype=F8, h_out=h)
    assert torch.equal(got[:, tokens], want) and torch.equal(s[:, tokens], ws)
    assert torch.equal(q.view(torch.uint8)[:, tokens], wq.view(torch.uint8))


def test_tensors_without_values_at_their_address_are_refused():
    """Zeros that autograd keeps without memory, fakes of tracing; parameters and plain subclasses have theirs."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    from paper_2511_22009_amd import quantize_f8, quantize_rows, residual_norm
    x = randn(gen(13), 4, 64)

    class Rows(torch.Tensor):
        pass
    for call in (quantize_rows, quantize_f8, lambda t: residual_norm(t, x, pre="rms"), lambda t: residual_norm(x, x, gate=t[0])):
        with pytest.raises(TypeError, match="zeros"):
            call(torch._efficientzerotensor((4, 64), device="cuda"))
        with FakeTensorMode() as mode:
            fake = mode.from_tensor(x)
        with pytest.raises(TypeError, match="fake"):
            call(fake)
        want = call(x)
        with torch.no_grad():
            for t in (torch.nn.Parameter(x), x.as_subclass(Rows)):
                for p, q in zip(call(t), want):
                    assert (p is None and q is None) or torch.equal(p.float(), q.float())
