"""The tables behind the tiles of e4m3 codes, compiled for the host from the header that the kernels include."""
import ast
import os
import re
import subprocess

from test_rules_cpu import CSRC, ROOT, _compiled
from test_rules_f8_cpu import F8_TILES, _f8_parts, _f8_tiles

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
