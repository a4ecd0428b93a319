"""The operators without a model, on the host: what they refuse, before any HIP call."""
import ctypes
import os
import subprocess

import pytest

from paper_2511_22009_amd import binding, load_library

P = ctypes.c_void_p
A16 = P(4096)                 # an address that is never read here: the calls are refused or empty
INVAL, OK = -1, 0


def rope(dims=(16, 16), layout=0, spread=0, theta=10000.0, axes=None):
    r = binding._Rope()
    r.axes = len(dims) if axes is None else axes
    for i, d in enumerate(dims[:4]):
        r.dims[i] = d
    r.layout, r.spread, r.theta = layout, spread, theta
    return r


def heads(n=4, tokens=8, dh=64, **kw):
    f = dict(in_=4096, out=8192, heads=n, in_row=tokens * n * dh, in_token=n * dh, in_head=dh, out_row=tokens * n * dh,
             out_token=n * dh, out_head=dh)
    f.update(kw)
    return binding._Heads(**f)


def quantize(x=A16, type=0, rows=4, cols=32, ldx=32, codes=A16, ldc=32, scale=A16):
    return load_library().sf_quantize_rows(x, type, rows, cols, ldx, codes, ldc, scale, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(codes=None), dict(scale=None), dict(type=2), dict(type=-1), dict(rows=-1),
                                 dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 20) + 1), dict(ldx=-8), dict(ldc=16),
                                 dict(ldc=40), dict(codes=P(4100))])
def test_quantize_rows_refuses(bad):
    assert quantize(**bad) == INVAL


def matmul(a=A16, lda=64, sa=A16, b=A16, ldb=64, sb=A16, bias=None, M=4, N=4, K=50, out=A16, ldo=4, type=0):
    return load_library().sf_matmul_i8(a, lda, sa, b, ldb, sb, bias, M, N, K, out, ldo, type, None)


@pytest.mark.parametrize("bad", [dict(a=None), dict(b=None), dict(sa=None), dict(sb=None), dict(out=None), dict(M=-1), dict(N=-1),
                                 dict(K=0), dict(K=-3), dict(K=131072), dict(lda=48), dict(ldb=48), dict(lda=65), dict(ldb=72),
                                 dict(lda=1 << 23), dict(ldb=1 << 23), dict(ldo=3), dict(type=2), dict(a=P(4104)), dict(b=P(4097))])
def test_matmul_i8_refuses(bad):
    assert matmul(**bad) == INVAL


def turn(h=None, type=0, rows=2, tokens=8, dh=64, r=None, pos=A16, pos_row=16, no_rope=False):
    h = heads() if h is None else h
    r = rope() if r is None else r
    return load_library().sf_rotate(ctypes.byref(h), type, rows, tokens, dh, None if no_rope else ctypes.byref(r), pos, pos_row, 0,
                                    None)


def qk(q=None, k=None, eps=1e-6, rows=2, tokens=8, dh=64, r=None, pos=A16):
    q = heads() if q is None else q
    return load_library().sf_qk_norm_rotate(ctypes.byref(q), None if k is None else ctypes.byref(k), None, None, eps, 0, rows,
                                            tokens, dh, None if r is None else ctypes.byref(r), pos, 16, None)


@pytest.mark.parametrize("bad", [dict(type=2), dict(rows=-1), dict(tokens=-1), dict(dh=63), dict(dh=0), dict(dh=258), dict(pos=None),
                                 dict(rows=1 << 16, tokens=1 << 15), dict(no_rope=True)])
def test_rotate_refuses_sizes(bad):
    assert turn(**bad) == INVAL


@pytest.mark.parametrize("bad", [dict(axes=0), dict(axes=5), dict(dims=(16, 15)), dict(dims=(64, 2)), dict(dims=(-2, 16)),
                                 dict(layout=3), dict(layout=-1), dict(spread=2), dict(theta=1.0), dict(theta=float("nan")),
                                 dict(theta=float("inf"))])
def test_rotate_refuses_plans(bad):
    assert turn(r=rope(**bad)) == INVAL


@pytest.mark.parametrize("bad", [dict(in_=None), dict(out=None), dict(out_row=0), dict(out_token=0), dict(out_head=0), dict(heads=-1),
                                 dict(heads=65536)])
def test_heads_that_cannot_be_written_are_refused(bad):
    assert turn(h=heads(**bad)) == INVAL
    assert qk(q=heads(**bad), r=rope()) == INVAL
    assert qk(k=heads(**bad), r=rope()) == INVAL


@pytest.mark.parametrize("eps", [-1.0, float("nan"), float("inf")])
def test_qk_norm_refuses_eps(eps):
    assert qk(eps=eps) == INVAL


def test_rotation_without_positions_is_refused():
    assert qk(r=rope(), pos=None) == INVAL


def test_empty_calls_are_no_work():
    assert quantize(rows=0) == OK and matmul(M=0) == OK and matmul(N=0) == OK
    assert turn(rows=0) == OK and turn(tokens=0) == OK and turn(h=heads(n=0)) == OK
    assert qk(q=heads(n=0), k=heads(n=0)) == OK


def test_null_head_tensors_are_refused():
    L = load_library()
    r = rope()
    assert L.sf_rotate(None, 0, 1, 1, 64, ctypes.byref(r), A16, 0, 0, None) == INVAL
    assert L.sf_qk_norm_rotate(None, None, None, None, 1e-6, 0, 1, 1, 64, None, None, 0, None) == INVAL


def test_python_refusals_without_a_gpu():
    torch = pytest.importorskip("torch")
    from paper_2511_22009_amd import Rotary, matmul_i8, qk_norm_rotate, quantize_rows, rotate
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        quantize_rows(x)
    with pytest.raises(TypeError):
        matmul_i8(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0])
    with pytest.raises(TypeError):
        rotate(torch.zeros(1, 1, 1, 8), torch.zeros(1, 1), Rotary([8]))
    with pytest.raises(TypeError):
        qk_norm_rotate(torch.zeros(1, 1, 1, 8), None)
    with pytest.raises(TypeError):
        quantize_rows([1.0])
    for dims in ([], [2, 2, 2, 2, 2], [3], [-2]):
        with pytest.raises(ValueError):
            Rotary(dims)
    with pytest.raises(ValueError):
        Rotary([8], layout="quarters")


TILES = r"""
#include <cstdio>
#include "sf_ops_rules.h"
int main() {
  const long sizes[] = {1, 2, 31, 64, 65, 129, 777, 1023, 4096, 16384, 70000, 1 << 20, 2147483647L};
  const long Ks[] = {1, 16, 100, 768, 4321, 131071};
  const auto rounds = [](long M, long N, long bm, long bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  for (int kind = 0; kind < 3; ++kind)  // a short epilogue, a long one, with the residual
    for (long M : sizes)
      for (long N : sizes)
        for (long K : Ks) {
          const auto t = sf::choose_gemm_i8_tile(M, N, K, kind > 0, kind == 2);
          if (t < sf::kI8Deep64 || t > sf::kI8Tile256x256) return std::printf("%ld %ld %ld: %d\n", M, N, K, (int)t), 1;
          // long epilogues: a single round of the tiles that a CU holds one of
          if (kind && t == sf::kI8Tile256x256) return 2;
          if (kind && t == sf::kI8Tile192x256 && rounds(M, N, 192, 256) > 256) return 2;
          if (kind && t == sf::kI8Deep128 && rounds(M, N, 128, 128) > 256) return 3;
          if (M > 60000 && N > 60000 && t < sf::kI8Tile128) return std::printf("%ld %ld %ld\n", M, N, K), 4;
          if (M <= 64 && N <= 4096 && t > sf::kI8Tile64) return std::printf("%ld %ld %ld\n", M, N, K), 5;
        }
  const auto at = [](long M, long N, long K) { return sf::choose_gemm_i8_tile(M, N, K, false, false); };
  if (at(4096, 2304, 768) != sf::kI8Tile192x256 || at(16384, 4608, 1152) != sf::kI8Tile256x256 ||
      at(16384, 1152, 4608) != sf::kI8Tile128x192 || at(1023, 777, 4321) != sf::kI8Deep64 || at(4096, 768, 4608) != sf::kI8Deep128)
    return 6;
  std::printf("ok\n");
  return 0;
}
"""


def test_choice_of_8_bit_tiles(tmp_path):
    """Every size gets a tile without an overflow, the largest ones the largest pairs, few rows
    a small one."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_22009_amd", "csrc")
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    with open(src, "w") as f:
        f.write(TILES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", csrc, src,
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)


def test_model_settings_need_a_model():
    L = load_library()
    assert L.sf_set_qk(None, None) == -3
    assert L.sf_set_int8(None, 1) == -3
