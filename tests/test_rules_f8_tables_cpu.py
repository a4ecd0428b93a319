"""The tables behind the tiles of e4m3 codes, compiled for the host from the header that the kernels include."""
import os
import re
import subprocess

from test_rules_cpu import CSRC, _compiled

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
