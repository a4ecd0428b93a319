"""Which tile a product of e4m3 codes takes, compiled for the host from the header that the kernels include."""
import ast
import os
import subprocess

from test_rules_cpu import ROOT, _compiled


F8_TILES = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads M N K codes exact gated, prints the tile and whether a kernel of it exists.
int main() {
  long M, N, K;
  int codes, exact, gated;
  while (scanf("%ld %ld %ld %d %d %d", &M, &N, &K, &codes, &exact, &gated) == 6) {
    const sf::F8Tile t = sf::choose_gemm_f8_tile(M, N, K, codes, exact, gated);
    printf("%d %d\n", (int)t, (int)sf::f8_has_tile(t, codes, exact));
  }
}
"""
F8_NAMES = ["few", "split32", "split32x4", "split64", "split64x4", "deep128", "tile128", "tile128x256", "tile256x256", "codes32", "codes64"]


def _f8_tiles(exe, calls):
    text = "".join("%d %d %d %d %d %d\n" % c for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()
    return [F8_NAMES[int(t)] for t in out[::2]], [int(v) for v in out[1::2]]


def test_f8_tiles_exist_for_every_size(tmp_path_factory):
    """The rule picks a tile that has a kernel for the output's kind, from the smallest sizes to the largest."""
    exe = _compiled(tmp_path_factory, "f8_tiles", F8_TILES)
    sizes = (1, 2, 16, 17, 32, 33, 64, 65, 300, 1152, 4096, 30000, 1 << 20, 8 << 20)
    calls = [(m, n, k, c, e, g) for m in sizes for n in sizes for k in (1, 128, 129, 4608, 1 << 20)
             for c, e, g in ((0, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 1))]
    names, exist = _f8_tiles(exe, calls)
    assert len(exist) == len(calls) and all(exist)
    for (m, _, _, _, _, _), name in zip(calls, names):
        assert name != "few" or m <= 32  # its workgroups hold no more rows


def test_f8_sizes_of_the_gpu_tests_reach_every_tile(tmp_path_factory):
    src = open(os.path.join(ROOT, "tests", "test_gpu_f8.py")).read()
    tree = ast.parse(src)
    sizes = next(ast.literal_eval(n.value) for n in tree.body if isinstance(n, ast.Assign) and n.targets[0].id == "SIZES")
    gated = next(ast.literal_eval(d.args[1]) for f in tree.body if isinstance(f, ast.FunctionDef) and f.name == "test_gated"
                 for d in f.decorator_list if d.args[0].value == "M,N,K")
    exe = _compiled(tmp_path_factory, "f8_sizes", F8_TILES)
    values = set(_f8_tiles(exe, [(*s, 0, 0, 0) for s in sizes])[0])
    assert values == {"few", "split32", "split64", "deep128", "tile128", "tile128x256", "tile256x256"}
    assert set(_f8_tiles(exe, [(*s, 0, 1, 0) for s in sizes])[0]) == {"few", "split32x4", "split64x4", "tile128"}
    both = [(m, 2 * n, k) for m, n, k in gated]
    assert set(_f8_tiles(exe, [(*s, 0, 0, 1) for s in both])[0]) == values
    assert set(_f8_tiles(exe, [(*s, 0, 1, 1) for s in both])[0]) == {"few", "split32x4", "split64x4", "tile128"}
    assert set(_f8_tiles(exe, [(*s, 1, 1, 1) for s in both])[0]) == {"codes32", "codes64"}


F8_PARTS = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads M N K codes exact, prints the rows and columns of the first part, and the costs of the whole and of both parts.
int main() {
  long M, N, K;
  int codes, exact;
  while (scanf("%ld %ld %ld %d %d", &M, &N, &K, &codes, &exact) == 5) {
    long rows, cols;
    sf::choose_gemm_f8_parts(M, N, K, codes, exact, rows, cols);
    const sf::F8Tiles t = sf::f8_tiles_of(codes, exact);
    const double whole = sf::cheapest_f8_tile(t.from, t.to, M, N, K).cost;
    double parts = sf::cheapest_f8_tile(t.from, t.to, rows, cols, K).cost;
    if (rows < M) parts += sf::cheapest_f8_tile(t.from, t.to, M - rows, N, K).cost;
    else if (cols < N) parts += sf::cheapest_f8_tile(t.from, t.to, M, N - cols, K).cost;
    printf("%ld %ld %.0f %.0f\n", rows, cols, whole, parts);
  }
}
"""


def _f8_parts(tmp_path_factory, calls):
    exe = _compiled(tmp_path_factory, "f8_parts", F8_PARTS)
    text = "".join("%d %d %d %d %d\n" % c for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()
    return [tuple(int(v) for v in out[4 * i:4 * i + 4]) for i in range(len(calls))]


def test_f8_parts_cover_the_product(tmp_path_factory):
    """A product is whole, or parted in rows or in columns, at whole blocks of weights, and then cheaper by the rule's own costs."""
    sizes = (1, 32, 33, 255, 256, 257, 640, 1152, 2049, 4200, 9000, 16384, 65537, 8 << 20)
    calls = [(m, n * g, k, c, e) for m in sizes for n in sizes for k in (1, 129, 1152, 4608, 1 << 20) for g, c, e in
             ((1, 0, 0), (1, 0, 1), (2, 0, 0), (2, 0, 1), (2, 1, 1))]
    parted = set()
    for (m, n, k, c, e), (rows, cols, whole, parts) in zip(calls, _f8_parts(tmp_path_factory, calls)):
        assert 0 < rows <= m and 0 < cols <= n
        if (rows, cols) == (m, n):
            continue
        assert whole >= 40000 and parts < whole and m > 32
        assert (rows < m) != (cols < n) and (cols == n or cols % 256 == 0)
        parted.add((c, e, rows < m))
    assert len(parted) >= 5


def test_f8_sizes_of_the_gpu_tests_are_parted(tmp_path_factory):
    tree = ast.parse(open(os.path.join(ROOT, "tests", "test_gpu_f8.py")).read())
    cases = next(ast.literal_eval(n.value) for n in tree.body if isinstance(n, ast.Assign) and n.targets[0].id == "PARTS")
    calls = [(m, n * (2 if gated else 1), k, int(kind == "f8"), int(kind != "bf16")) for m, n, k, kind, gated, _ in cases]
    for call, case, (rows, cols, _, _) in zip(calls, cases, _f8_parts(tmp_path_factory, calls)):
        assert (rows < call[0], cols < call[1]) == (case[5] == "rows", case[5] == "cols"), case
    assert {(c[3], c[4], c[5]) for c in cases} == {(k, g, p) for k, g in (("bf16", False), ("fp32", False), ("bf16", True), ("fp32", True),
                                                                         ("f8", True)) for p in ("rows", "cols")}
