"""The operators in 8-bit floating point and the norms around a block where their ranges end."""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
from f8_util import BF16, F8, FP32  # noqa: E402

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
