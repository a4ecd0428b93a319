"""What the operators on torch tensors refuse of tensors that are differentiated, or that have no values at their address, on the
host: the tensors are fakes of a GPU's, which every call refuses last."""
import pytest

torch = pytest.importorskip("torch")

import torch.autograd.forward_ad as fw  # noqa: E402
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

F8 = torch.float8_e4m3fn


def inputs():
    """Every tensor that a call takes, by name."""
    e = lambda *shape, dtype=torch.float32: torch.empty(shape, device="cuda:0", dtype=dtype)  # noqa: E731
    return dict(x=e(4, 32), i8=e(4, 32, dtype=torch.int8), i8_scale=e(4), h=e(2, 3, 4, 64), pos=e(3, 2), gain=e(64), out=e(4, 4),
                f8=e(4, 32, dtype=F8), row_scale=e(4, 1), w=e(4, 32, dtype=F8), w_scale=e(1, 1), bias=e(4), rows=e(2, 3, 32), y=e(2, 3, 32),
                per=e(2, 32), dims=e(32))


def calls(t):
    """(name, call with that tensor replaced) for every operator and each of its floating tensors."""
    from paper_2511_22009_amd import (Rotary, gated_matmul_f8, matmul_f8, matmul_i8, qk_norm_rotate, quantize_f8, quantize_rows,
                                      residual_norm, rotate)
    r = Rotary([32, 32])
    forms = [
        (("x",), lambda x: quantize_rows(x)), (("i8_scale",), lambda s: quantize_rows(t["x"], scale=s)),
        (("i8_scale", "i8_scale", "bias", "out"), lambda sa, sb, b, o: matmul_i8(t["i8"], sa, t["i8"], sb, b, out=o)),
        (("h", "pos", "h"), lambda x, p, o: rotate(x, p, r, out=o)),
        (("h", "h", "gain", "gain", "pos", "h", "h"), lambda q, k, a, b, p, o, u: qk_norm_rotate(q, k, a, b, p, r, out=(o, u))),
        (("x", "row_scale"), lambda x, s: quantize_f8(x, scale=s)),
        (("row_scale", "w_scale", "bias", "out"), lambda sa, sb, b, o: matmul_f8(t["f8"], sa, t["w"], sb, b, out=o)),
        (("row_scale", "w_scale", "w_scale", "bias", "bias", "out"),
         lambda sa, sg, su, g, u, o: gated_matmul_f8(t["f8"], sa, t["w"], sg, t["w"], su, g, u, out=o)),
        (("rows", "y", "per", "dims", "dims", "per", "per", "rows", "y"),
         lambda h, y, g, a, b, c, s, ho, o: residual_norm(h, y, g, "rms", a, 1.0, "layer", b, c, s, h_out=ho, out=o)),
    ]
    for names, call in forms:
        for n, name in enumerate(names):
            def replaced(f, names=names, call=call, n=n):
                return call(*(f(t[m]) if i == n else t[m] for i, m in enumerate(names)))
            yield name, replaced


def passes_its_checks(call):
    """Whether a call passes all of them but the last, that a fake has no values at its address."""
    with pytest.raises(TypeError) as e:
        call()
    return "a fake tensor" in str(e.value)


@pytest.fixture
def fakes():
    pytest.importorskip("paper_2511_22009_amd.operators")
    with FakeTensorMode(allow_non_fake_inputs=True):
        yield inputs()


def test_every_call_passes_its_checks_as_it_is(fakes):
    for name, call in calls(fakes):
        assert passes_its_checks(lambda: call(lambda t: t)), name


def test_tensors_that_require_grad_are_refused(fakes):
    for name, call in calls(fakes):
        with pytest.raises(TypeError, match="requires grad"):
            call(lambda t: t.detach().clone().requires_grad_())
        with torch.no_grad():
            assert passes_its_checks(lambda: call(lambda t: t.detach().clone().requires_grad_())), name


def test_tensors_with_a_forward_mode_tangent_are_refused(fakes):
    """The tangent would be dropped without a word, gradients recorded or not."""
    for name, call in calls(fakes):
        for grad in (True, False):
            with torch.set_grad_enabled(grad), fw.dual_level():
                with pytest.raises(TypeError, match="tangent"):
                    call(lambda t: fw.make_dual(t, torch.ones_like(t)))
                assert passes_its_checks(lambda: call(lambda t: fw.unpack_dual(fw.make_dual(t, torch.ones_like(t))).primal)), name
        assert passes_its_checks(lambda: call(lambda t: t)), name


def test_fakes_are_refused_whose_address_is_not_null(fakes):
    """Views of fakes have addresses of a few bytes, which a kernel would read."""
    from paper_2511_22009_amd import quantize_f8, quantize_rows, residual_norm
    for call in (lambda: quantize_rows(fakes["x"][1:]), lambda: quantize_f8(fakes["x"][2:]), lambda: residual_norm(fakes["rows"][1:], fakes["y"][1:])):
        with pytest.raises(TypeError, match="fake"):
            call()
