"""Which tile a product of e4m3 codes takes, compiled for the host from the header that the kernels include."""
import ast
import os
import subprocess

from test_rules_cpu import ROOT, _compiled


F8_TILES = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads M N K codes exact, prints the tile and whether a kernel of it exists.
int main() {
  long M, N, K;
  int codes, exact;
  while (scanf("%ld %ld %ld %d %d", &M, &N, &K, &codes, &exact) == 5) {
    const sf::F8Tile t = sf::choose_gemm_f8_tile(M, N, K, codes, exact);
    printf("%d %d\n", (int)t, (int)sf::f8_has_tile(t, codes, exact));
  }
}
"""
F8_NAMES = ["few", "split32", "split32x4", "split64", "split64x4", "deep128", "tile128", "tile128x256", "tile256x256", "codes32", "codes64"]


def _f8_tiles(exe, calls):
    text = "".join("%d %d %d %d %d\n" % c for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()
    return [F8_NAMES[int(t)] for t in out[::2]], [int(v) for v in out[1::2]]


def test_f8_tiles_exist_for_every_size(tmp_path_factory):
    """The rule picks a tile that has a kernel for the output's kind, from the smallest sizes to the largest."""
    exe = _compiled(tmp_path_factory, "f8_tiles", F8_TILES)
    sizes = (1, 2, 16, 17, 32, 33, 64, 65, 300, 1152, 4096, 30000, 1 << 20, 8 << 20)
    calls = [(m, n, k, c, e) for m in sizes for n in sizes for k in (1, 128, 129, 4608, 1 << 20) for c, e in ((0, 0), (0, 1), (1, 1))]
    names, exist = _f8_tiles(exe, calls)
    assert len(exist) == len(calls) and all(exist)
    for (m, n, k, c, e), name in zip(calls, names):
        assert name != "few" or m <= 32  # its workgroups hold no more rows


def test_f8_sizes_of_the_gpu_tests_reach_every_tile(tmp_path_factory):
    src = open(os.path.join(ROOT, "tests", "test_gpu_f8.py")).read()
    tree = ast.parse(src)
    sizes = next(ast.literal_eval(n.value) for n in tree.body if isinstance(n, ast.Assign) and n.targets[0].id == "SIZES")
    gated = next(ast.literal_eval(d.args[1]) for f in tree.body if isinstance(f, ast.FunctionDef) and f.name == "test_gated"
                 for d in f.decorator_list if d.args[0].value == "M,N,K")
    exe = _compiled(tmp_path_factory, "f8_sizes", F8_TILES)
    values = set(_f8_tiles(exe, [(*s, 0, 0) for s in sizes])[0])
    assert values == {"few", "split32", "split64", "deep128", "tile128", "tile128x256", "tile256x256"}
    assert set(_f8_tiles(exe, [(*s, 0, 1) for s in sizes])[0]) == {"few", "split32x4", "split64x4", "tile128"}
    both = [(m, 2 * n, k) for m, n, k in gated]
    assert set(_f8_tiles(exe, [(*s, 0, 0) for s in both])[0]) == values
    assert set(_f8_tiles(exe, [(*s, 0, 1) for s in both])[0]) == {"few", "split32x4", "split64x4", "tile128"}
    assert set(_f8_tiles(exe, [(*s, 1, 1) for s in both])[0]) == {"codes32", "codes64"}
