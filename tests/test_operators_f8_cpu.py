"""The operators in 8-bit floating point and the norms around a block, on the host: what they refuse, before any HIP call."""
import ctypes

import pytest

from paper_2511_22009_amd import binding, load_library

P = ctypes.c_void_p
A16 = P(4096)                 # addresses that are never read here: the calls are refused or empty
INVAL, OK = -1, 0


def codes(at=4096, ld=64, scale=8192, scale_row=1, scale_block=4):
    return binding._Codes(at, ld, scale, scale_row, scale_block)


def quantize(x=P(1 << 20), type=0, rows=4, cols=200, ldx=200, block_rows=1, codes=A16, ldc=208, scale=P(8192), scale_row=1, scale_block=4):
    return load_library().sf_quantize_f8(x, type, rows, cols, ldx, block_rows, codes, ldc, scale, scale_row, scale_block, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(codes=None), dict(scale=None), dict(type=2), dict(type=-1), dict(rows=-1),
                                 dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 20) + 1), dict(ldx=-8), dict(ldc=192), dict(ldc=201),
                                 dict(codes=P(4100)), dict(block_rows=0), dict(block_rows=2), dict(block_rows=127), dict(scale_row=0),
                                 dict(scale_block=0), dict(scale_row=-1), dict(scale_block=-4), dict(codes=P(1 << 20)),
                                 dict(scale=P(1 << 20))])
def test_quantize_refuses(bad):
    assert quantize(**bad) == INVAL


def matmul(a=None, b=None, bias=None, M=4, N=4, K=50, out=P(1 << 20), ldo=4, type=0, no=None):
    a, b = codes() if a is None else a, codes(at=1 << 16) if b is None else b
    return load_library().sf_matmul_f8(None if no == "a" else ctypes.byref(a), None if no == "b" else ctypes.byref(b), bias, M, N, K, out,
                                       ldo, type, None)


def gated(a=None, gate=None, up=None, act=0, M=4, N=200, K=50, out=P(1 << 20), ldo=208, type=2, out_scale=P(1 << 24), scale_row=1,
          scale_block=4, no=None):
    a, gate, up = (codes(at=n << 16) if c is None else c for n, c in ((1, a), (2, gate), (3, up)))
    refs = [None if no == n else ctypes.byref(c) for n, c in (("a", a), ("gate", gate), ("up", up))]
    return load_library().sf_gated_matmul_f8(*refs, None, None, act, M, N, K, out, ldo, type, out_scale, scale_row, scale_block, None)


CODES = [dict(at=None), dict(at=4104), dict(ld=48), dict(ld=65), dict(ld=1 << 23), dict(scale=None), dict(scale_row=-1),
         dict(scale_row=1 << 20), dict(scale_block=-1)]


@pytest.mark.parametrize("bad", CODES)
def test_products_refuse_codes(bad):
    assert matmul(a=codes(**bad)) == INVAL
    assert matmul(b=codes(**bad)) == INVAL
    for n in ("a", "gate", "up"):
        assert gated(**{n: codes(**bad)}) == INVAL


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=-1), dict(K=0), dict(K=-3), dict(K=(1 << 20) + 1), dict(out=None), dict(ldo=3),
                                 dict(type=2), dict(type=3), dict(type=-1), dict(no="a"), dict(no="b"), dict(out=P(4096)),
                                 dict(out=P(1 << 16))])
def test_matmul_refuses(bad):
    assert matmul(**bad) == INVAL


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=-1), dict(K=0), dict(out=None), dict(ldo=192), dict(ldo=201), dict(out=P((1 << 20) + 8)),
                                 dict(type=3), dict(type=-1), dict(act=2), dict(act=-1), dict(no="a"), dict(no="gate"), dict(no="up"),
                                 dict(out_scale=None), dict(scale_row=0), dict(scale_block=0), dict(scale_row=-1), dict(out=P(3 << 16)),
                                 dict(type=0, ldo=199)])
def test_gated_refuses(bad):
    assert gated(**bad) == INVAL


def rows(samples=2, tokens=3, dims=200, **kw):
    f = dict(samples=samples, tokens=tokens, dims=dims, h=1 << 20, h_type=1, h_sample=tokens * dims, h_token=dims, y=2 << 20, y_type=0,
             y_sample=tokens * dims, y_token=dims, h_out=3 << 20, h_out_sample=tokens * dims, h_out_token=dims, post=1, residual_scale=1.0,
             pre=2, eps=1e-6, out=4 << 20, out_type=2, out_sample=tokens * 208, out_token=208, out_scale=5 << 20, out_scale_sample=6,
             out_scale_token=2, out_scale_block=1)
    f.update(kw)
    return load_library().sf_residual_norm(ctypes.byref(binding._BlockRows(**f)), None)


@pytest.mark.parametrize("bad", [dict(samples=-1), dict(tokens=-1), dict(samples=1 << 16, tokens=1 << 15), dict(dims=0), dict(dims=16385),
                                 dict(h=None), dict(y=None), dict(h_out=None), dict(h_type=2), dict(y_type=2), dict(h_type=-1),
                                 dict(out_type=3), dict(post=3), dict(post=-1), dict(pre=3), dict(pre=-1),
                                 dict(residual_scale=float("nan")), dict(residual_scale=float("inf")), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(h_out_sample=0), dict(h_out_token=0),
                                 dict(h_out=2 << 20), dict(h_out=1 << 20, h_out_token=100), dict(h_out=1 << 20, h_out_sample=1000),
                                 dict(out_sample=0), dict(out_token=0), dict(out=1 << 20), dict(out=2 << 20), dict(out=3 << 20),
                                 dict(out_scale=None), dict(out_token=200), dict(out_sample=1000), dict(out=(4 << 20) + 8),
                                 dict(out_scale_sample=0), dict(out_scale_token=0), dict(out_scale_block=0)])
def test_residual_norm_refuses(bad):
    assert rows(**bad) == INVAL


def test_residual_norm_refuses_nothing_at_all():
    assert load_library().sf_residual_norm(None, None) == INVAL


def test_empty_calls_are_no_work():
    assert quantize(rows=0, x=None, codes=None, scale=None) == OK
    assert matmul(M=0, out=None) == OK and matmul(N=0, out=None) == OK
    assert gated(M=0, out=None) == OK and gated(N=0, out=None) == OK
    assert rows(samples=0, h=None) == OK and rows(tokens=0, h=None) == OK


def test_structs_are_laid_out_as_the_header_has_them(tmp_path):
    import os
    import subprocess

    from conftest import ROOT
    names = {"sf_codes": binding._Codes, "sf_block_rows": binding._BlockRows}
    src = tmp_path / "s.c"
    body = "".join(f'printf("%zu ", sizeof({n}));' + "".join(f'printf("%zu ", offsetof({n}, {f[0]}));' for f in c._fields_) for n, c in names.items())
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "streamflow.h"\nint main(void) {{ {body} return 0; }}\n')
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = [v for c in names.values() for v in (ctypes.sizeof(c), *(getattr(c, f[0]).offset for f in c._fields_))]
    assert got == want


def test_python_refuses_names_and_types():
    torch = pytest.importorskip("torch")
    from paper_2511_22009_amd import gated_matmul_f8, matmul_f8, quantize_f8, residual_norm
    x = torch.zeros(4, 4)
    with pytest.raises(TypeError, match="CUDA"):
        quantize_f8(x)
    with pytest.raises(TypeError, match="CUDA"):
        matmul_f8(x, x, x, x)
    with pytest.raises(TypeError, match="dtype"):
        matmul_f8(x, x, x, x, dtype=torch.float8_e4m3fn)
    with pytest.raises(TypeError, match="dtype"):
        gated_matmul_f8(x, x, x, x, x, x, dtype=torch.float16)
    with pytest.raises(ValueError, match="activation"):
        gated_matmul_f8(x, x, x, x, x, x, activation="relu")
    with pytest.raises(TypeError, match="CUDA"):
        residual_norm(x, x)
    for kw in (dict(post="batch"), dict(pre="batch"), dict(post=1), dict(pre=[])):
        with pytest.raises(ValueError, match="post|pre"):
            residual_norm(x, x, **kw)
    with pytest.raises(TypeError, match="dtype"):
        residual_norm(x, x, dtype=None)
