"""The operators' plans and the package's names, on the host."""
import copy
import ctypes
import pickle
import subprocess
import sys

import pytest

from conftest import ROOT


def plan(r):
    """What the library would read at the address that a call passes."""
    from paper_2511_22009_amd import binding
    s = r._struct
    assert r._address == ctypes.addressof(s)
    at = binding._Rope.from_address(ctypes.addressof(s))
    return at.axes, tuple(at.dims), at.layout, at.spread, at.theta


@pytest.mark.parametrize("way", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r)),
                                 lambda r: copy.deepcopy({"rotary": [r]})["rotary"][0]], ids=["copy", "deepcopy", "pickle", "nested"])
def test_copies_of_a_plan_have_memory_of_their_own(way):
    """A plan's address goes to the library, so a copy passes its own, which lives as long as it."""
    pytest.importorskip("torch")
    from paper_2511_22009_amd import Rotary
    r = Rotary((16, 24, 0), theta=500.0, layout="axis_halves", spread=True)
    c = way(r)
    assert (c.dims, c.theta, c.layout, c.spread) == (r.dims, r.theta, r.layout, r.spread)
    want = plan(r)
    assert c._address != r._address
    del r
    assert plan(c) == want


def run(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


NAMES = ["Rotary", "matmul_i8", "qk_norm_rotate", "quantize_rows", "rotate"]


@pytest.mark.parametrize("missing", ["torch", "paper_2511_22009_amd._operators"])
def test_every_name_of_the_package_without_torch_or_the_operators_binding(missing):
    """`import *` gives what can be loaded: all but the operators, which need both; these say so."""
    got = run(f"import sys; sys.modules[{missing!r}] = None\n"
              "from paper_2511_22009_amd import *\n"
              "import paper_2511_22009_amd as p\n"
              "assert Model is p.Model and load_library() is not None\n"
              "try:\n    p.rotate\nexcept ImportError: print('refused')\n"
              "print(*(n for n in dir() if not n.startswith('_')))")
    assert got[0] == "refused" and "Model" in got and "library_symbols" in got and not set(NAMES) & set(got)


def test_every_name_of_the_package():
    pytest.importorskip("torch")
    got = run("from paper_2511_22009_amd import *\nprint(*(n for n in dir() if not n.startswith('_')))")
    assert set(NAMES) < set(got) and "Model" in got


def test_importing_the_package_needs_no_torch():
    assert run("import paper_2511_22009_amd, sys\nprint('torch' in sys.modules)") == ["False"]


@pytest.mark.parametrize("bad", [(16, 16), {"dims": (16, 16)}, 5, object()])
def test_set_qk_takes_a_plan_and_nothing_else(bad):
    from paper_2511_22009_amd import Model, load_library
    load_library()
    m = Model.__new__(Model)                     # no handle: the library answers that none is loaded
    m._h, m.info = None, dict(L=2, D=128, heads=4)
    with pytest.raises(TypeError, match="rotary"):
        m.set_qk(rotary=bad)
    pytest.importorskip("torch")
    from paper_2511_22009_amd import Rotary, SFError
    for good in (None, Rotary([16, 16])):
        with pytest.raises(SFError) as e:
            m.set_qk(rotary=good)
        assert e.value.code == -3


PAIRS = r"""
#include <cstdio>
#include <cstdlib>
#include "sf_ops_rules.h"
// widths, MLP widths and token rows; prints the tiles of QKV, GELU and residual
int main(int n, char** v) {
  for (int i = 1; i + 2 < n; i += 3) {
    const long D = std::atol(v[i]), F = std::atol(v[i + 1]), M = std::atol(v[i + 2]);
    std::printf("q%d g%d r%d r%d\n", (int)sf::choose_gemm_i8_tile(M, 3 * D, D, true, false), (int)sf::choose_gemm_i8_tile(M, F, D, true, false),
                (int)sf::choose_gemm_i8_tile(M, D, D, true, true), (int)sf::choose_gemm_i8_tile(M, D, F, true, true));
  }
  return 0;
}
"""


def test_gpu_cases_of_8_bit_projections_take_every_tile(tmp_path):
    """Every tile that a projection with an epilogue of its own can take is one that a case of
    test_gpu_int8_tiles.py takes: all but the largest, for each of the three epilogues."""
    import os
    pytest.importorskip("torch")
    import workloads
    from test_gpu_int8_tiles import SHAPES
    csrc = os.path.join(ROOT, "paper_2511_22009_amd", "csrc")
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    with open(src, "w") as f:
        f.write(PAIRS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", csrc, src, "-o", exe], check=True)

    def tiles(shapes):
        out = subprocess.run([exe, *(str(v) for s in shapes for v in s)], capture_output=True, text=True, check=True).stdout
        return set(out.split())
    got = tiles([(c.D, c.mlp, c.N * rows) for c, rows in SHAPES])
    assert got == {k + str(t) for k in "qgr" for t in range(6)}
    # the networks of the workloads, with one to all of their rows, and a wide sweep, reach no others
    named = [workloads.get_config(n) for n in workloads.CONFIGS]
    assert tiles([(c.D, c.mlp, c.N * r) for c in named for r in range(1, c.rows + 1)]) <= got
    assert tiles([(D, m * D, M) for D in range(64, 2049, 64) for m in (1, 2, 4) for M in (1, 64, 300, 1024, 4096, 16384, 65536)]) <= got


TILE = r"""
#include <cstdio>
#include <cstdlib>
#include "sf_ops_rules.h"
int main(int n, char** v) {
  for (int i = 1; i + 2 < n; i += 3) std::printf("%d ", (int)sf::choose_gemm_i8_tile(std::atol(v[i]), std::atol(v[i + 1]), std::atol(v[i + 2]), false, false));
  return 0;
}
"""


def test_gpu_cases_of_equal_bits_compare_different_tiles(tmp_path):
    """Whole products in the tiles from 128 x 128 on, parts of them in 64 x 64."""
    import os
    pytest.importorskip("torch")
    from test_gpu_operators_edges import test_products_have_the_same_bits_in_every_tile as t
    sizes = next(m for m in t.pytestmark if m.args[0] == "M,N,K").args[1]
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    with open(src, "w") as f:
        f.write(TILE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2511_22009_amd", "csrc"), src, "-o", exe], check=True)

    def tiles(shapes):
        return [int(w) for w in subprocess.run([exe, *(str(v) for s in shapes for v in s)], capture_output=True, text=True, check=True).stdout.split()]
    whole = tiles(sizes)
    assert set(whole) == {2, 3, 4, 5, 6}
    assert max(tiles([s for M, N, K in sizes for s in ((64, N, K), (M, 64, K))])) <= 1


def heads(at, out, n=4, tokens=8, dh=64, row=None, token=None, head=None):
    from paper_2511_22009_amd import binding
    s = (tokens * n * dh, n * dh, dh)
    return binding._Heads(at, out, n, *s, s[0] if row is None else row, s[1] if token is None else token, s[2] if head is None else head)


def turned(q, k=None, rows=2, tokens=8):
    """The status of a call that is refused (addresses are never read): without a GPU one that is not ends at its launch."""
    from paper_2511_22009_amd import load_library
    return load_library().sf_qk_norm_rotate(ctypes.byref(q), None if k is None else ctypes.byref(k), None, None, 1e-6, 0, rows, tokens,
                                            64, None, None, 0, None)


@pytest.mark.parametrize("other", [dict(row=1 << 20), dict(token=64, head=512), dict(head=128)])
def test_results_over_their_inputs_with_other_strides_are_refused(other):
    """A head would be written over one that is still to be read."""
    assert turned(heads(4096, 4096, **other)) == -1
    assert turned(heads(4096, 8192), heads(1 << 20, 1 << 20, **other)) == -1


def test_results_over_the_other_tensors_are_refused():
    a, b, c, d = (1 << 20) * 1, (1 << 20) * 2, (1 << 20) * 3, (1 << 20) * 4
    for q, k in (((a, b), (b, a)), ((a, c), (b, c)), ((a, b), (b, c)), ((a, c), (b, a)), ((a, a), (a, a)), ((a, a), (a, d))):
        assert turned(heads(*q), heads(*k)) == -1
