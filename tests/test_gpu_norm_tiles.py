"""Every kernel of the norms around a block, with few rows and with many, in place and not, against plain 64-bit forms."""
import pytest

pytestmark = pytest.mark.gpu

from gpu_util import torch  # noqa: E402
from f8_util import BF16, F8, FP32, gen  # noqa: E402
from test_gpu_f8 import check_rows, flat, make_rows  # noqa: E402

ids = lambda v: str(v).replace("torch.", "")  # noqa: E731

# Samples, tokens, dims. From 2048 rows on a wavefront takes a row of up to 1280 dims, and a workgroup several rows in turn, the last
# of a sample fewer than the others.
FEW = [(2, 30, 200), (3, 41, 255), (2, 9, 768), (1, 17, 1022), (2, 5, 1276), (3, 5, 1279), (1, 6, 4096), (2, 3, 4095), (1, 3, 8188),
       (2, 2, 8189), (1, 2, 16380), (1, 3, 16381)]
MANY = [(1, 9000, 64), (7, 599, 256), (3, 700, 260), (1, 5003, 768), (2, 2049, 772), (5, 411, 1024), (2, 1030, 1028), (3, 1367, 1152),
        (1, 4099, 1280), (9, 231, 516), (2, 1200, 253), (3, 701, 771), (2, 1100, 1281), (1, 2100, 2052), (1, 2051, 5001)]


@pytest.mark.parametrize("dtype", [BF16, FP32, F8], ids=ids)
@pytest.mark.parametrize("hd,yd", [(FP32, BF16), (BF16, FP32), (FP32, FP32), (BF16, BF16)], ids=ids)
@pytest.mark.parametrize("S,T,D", FEW + MANY)
def test_norms(S, T, D, hd, yd, dtype):
    """And over h itself the same bits: a workgroup reads its next row of h before it writes this one's."""
    from paper_2511_22009_amd import residual_norm
    g = gen(S * T + D)
    n = (S + T + D + (hd == FP32) + 2 * (yd == FP32)) % 4
    post, pre = (("rms", "layer"), ("layer", "rms"), ("none", "layer"), ("rms", "none"))[n]
    h, y, v = make_rows(g, S, T, D, hd, yd, ("sample", "channel", None)[(n + T) % 3], n % 2 == 0, n != 3)
    want = check_rows(h, y, v, post, pre, (1.0, 0.5)[n % 2], dtype)
    got = residual_norm(h, y, post=post, pre=pre, residual_scale=(1.0, 0.5)[n % 2], dtype=dtype, h_out=h, **v)
    assert got[0] is h
    for a, b in zip(flat(got), flat(want)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("S,T,D", FEW + MANY)
def test_codes_are_those_of_the_values(S, T, D):
    """As codes, the bits that quantize_f8 gives of the same call's fp32 values: the same arithmetic up to them."""
    from paper_2511_22009_amd import quantize_f8, residual_norm
    h, y, v = make_rows(gen(S + T + D), S, T, D, FP32, BF16, "sample", True, True)
    for post, pre in (("rms", "layer"), ("layer", "rms")):
        values = residual_norm(h, y, post=post, pre=pre, dtype=FP32, **v)[1]
        q, s = residual_norm(h, y, post=post, pre=pre, dtype=F8, **v)[1]
        want, scale = quantize_f8(values.flatten(0, 1))
        assert torch.equal(s.flatten(0, 1), scale)
        assert torch.equal(q.flatten(0, 1).view(torch.uint8), want.view(torch.uint8))
