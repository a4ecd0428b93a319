"""The tables behind the tiles of e4m3 codes, compiled for the host from the header that the kernels include."""
import ast
import os
import re
import subprocess

from test_rules_cpu import CSRC, ROOT, _compiled
from test_rules_f8_cpu import F8_NAMES, F8_TILES, _f8_parts, _f8_tiles

TABLES = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Every tile that a kind of output may take by its cost, its sizes, and whether a kernel of it exists.
int main() {
  for (int codes = 0; codes < 2; ++codes)
    for (int exact = codes; exact < 2; ++exact) {
      const sf::F8Tiles t = sf::f8_tiles_of(codes, exact);
      for (const sf::F8Cost* c = t.from; c != t.to; ++c)
        printf("%d %d %d %d %d\n", (int)c->tile, c->bm, c->bn, c->per, (int)sf::f8_has_tile(c->tile, codes, exact));
    }
}
"""


def test_every_tile_of_the_tables_has_a_kernel(tmp_path_factory):
    """Of its sizes, and for the kind of output whose table names it: the launch refuses any other."""
    out = subprocess.run([_compiled(tmp_path_factory, "f8_tables", TABLES)], capture_output=True, text=True, check=True).stdout
    rows = [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    rules = open(os.path.join(CSRC, "sf_ops_rules.h")).read()
    names = re.findall(r"kF8\w+", re.search(r"enum F8Tile \{(.*?)\}", rules, re.S).group(1))
    kernels = open(os.path.join(CSRC, "k_gemm_f8.hip")).read()
    sizes = {m[0]: (int(m[1]), int(m[2])) for m in re.findall(r"X\((kF8\w+), (\d+), (\d+),", kernels)}
    assert len(rows) == 11 and set(sizes) == set(names) - {"kF8Few"}
    for tile, bm, bn, per, exists in rows:
        assert exists and sizes[names[tile]] == (bm, bn) and per in (1, 2)


def test_sizes_of_the_tests_of_sums_take_every_tile(tmp_path_factory):
    """And products in two launches, in rows or in columns; where codes and values are compared bit for bit, values are in whole tiles."""
    tree = ast.parse(open(os.path.join(ROOT, "tests", "test_gpu_f8_sums.py")).read())
    sizes = {n.targets[0].id: ast.literal_eval(n.value) for n in tree.body if isinstance(n, ast.Assign) and n.targets[0].id in ("PRODUCTS", "GATED")}
    tiles, parts = _compiled(tmp_path_factory, "sums_tiles", F8_TILES), []

    def taken(of, codes, exact, gated):
        calls = [(m, n * (2 if gated else 1), *(k or [1152]), codes, exact) for m, n, *k in of]
        parts.extend(rows < m or cols < n for (m, n, *_), (rows, cols, _, _) in zip(calls, _f8_parts(tmp_path_factory, calls)))
        return set(_f8_tiles(tiles, [(*c, gated) for c in calls])[0])
    assert taken(sizes["PRODUCTS"], 0, 0, 0) | taken(sizes["GATED"], 0, 0, 1) == {
        "few", "split32", "split64", "deep128", "tile128", "tile128x256", "tile256x256"}
    assert taken(sizes["PRODUCTS"], 0, 1, 0) == taken(sizes["GATED"], 0, 1, 1) == {"few", "split32x4", "split64x4", "tile128"}
    assert taken(sizes["GATED"], 1, 1, 1) == {"codes32", "codes64"} and any(parts)
    whole = next(ast.literal_eval(d.args[1]) for f in tree.body if isinstance(f, ast.FunctionDef) and f.name == "test_codes_are_those_of_the_values"
                 for d in f.decorator_list if d.args[0].value == "M,N,K")
    calls = [(m, 2 * n, k, 0, 1) for m, n, k in whole]
    assert set(_f8_tiles(tiles, [(*c, 1) for c in calls])[0]) == {"tile128"}
    assert all((rows, cols) == c[:2] for c, (rows, cols, _, _) in zip(calls, _f8_parts(tmp_path_factory, calls)))


GRIDS = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads M N, prints the rows and columns of a call's launches.
int main() {
  long long M, N;
  while (scanf("%lld %lld", &M, &N) == 2)
    printf("%lld %lld\n", (long long)sf::f8_most_rows(N), (long long)sf::kF8MostColumns);
}
"""


def test_grids_at_the_ends_of_the_ranges_hold_less_than_2_to_the_32_threads(tmp_path_factory):
    """Whole launches and what is left of them, up to the largest sizes that a call takes, in parts and tiles as the rule has them."""
    top = (1 << 31) - 1
    sizes = (1, 15, 16, 17, 32, 33, 64, 257, 1152, 8191, 8192, 8193, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 30) + 3, top)
    calls = [(m, n) for m in sizes for n in sizes]
    out = [int(v) for v in subprocess.run([_compiled(tmp_path_factory, "grids", GRIDS)], input="".join("%d %d\n" % c for c in calls),
                                          capture_output=True, text=True, check=True).stdout.split()]
    launches = set()
    for (m, n), rows, cols in zip(calls, out[::2], out[1::2]):
        assert rows >= 8192 and rows <= 1 << 23 and rows % 256 == 0 and cols % 128 == 0
        launches |= {(r, c) for r in {min(m, rows), m % rows} for c in {min(n, cols), n % cols} if r and c}
    kernels = open(os.path.join(CSRC, "k_gemm_f8.hip")).read()
    tile = {m[0]: [int(v) for v in m[1].split(",")] for m in re.findall(r"X\((kF8\w+), ([\d, ]+)\)", kernels)}
    names = re.findall(r"kF8\w+", re.search(r"enum F8Tile \{(.*?)\}", open(os.path.join(CSRC, "sf_ops_rules.h")).read(), re.S).group(1))
    tiles = _compiled(tmp_path_factory, "grid_tiles", F8_TILES)
    kinds = ((0, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 1))
    whole = [(r, c, k, *kind) for r, c in sorted(launches) for k in (1, 128, 1152, 4096, 1 << 20) for kind in kinds]
    parts = _f8_parts(tmp_path_factory, [(r, c * (1 + g), k, codes, exact) for r, c, k, codes, exact, g in whole])
    grids = set()
    for (r, c, k, codes, exact, g), (rows, cols, _, _) in zip(whole, parts):
        cols //= 1 + g
        grids |= {(rows, cols, k, codes, exact, g)}
        if rows < r:
            grids.add((r - rows, c, k, codes, exact, g))
        elif cols < c:
            grids.add((r, c - cols, k, codes, exact, g))
    grids = sorted(grids)
    taken = _f8_tiles(tiles, [(r, c * (1 + g), k, codes, exact, g) for r, c, k, codes, exact, g in grids])[0]
    index = {n: names[i] for i, n in enumerate(F8_NAMES)}
    for (r, c, k, codes, exact, g), name in zip(grids, taken):
        if name == "few":
            groups, threads = -(-c // 16), 64 * (8 if k >= 4096 else 4)
        else:
            bm, bn, wm, wn, wk = tile[index[name]][:5]
            groups, threads = -(-r // bm) * -(-c // (bn // 2 if g else bn)), wm * wn * wk * 64
        assert groups * threads < 1 << 32, (r, c, k, name)
