"""The operators in 8-bit floating point and the norms around a block where their ranges end."""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
from f8_util import BF16  # noqa: E402


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
