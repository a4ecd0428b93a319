"""How the rows around a block are shared out over launches and workgroups, compiled for the host from the header that the
kernels include."""
import ast
import os
import re
import subprocess

from test_rules_cpu import CSRC, ROOT, _compiled

PARTS = r"""
#include <cstdio>
#include <cstdlib>
#include "sf_ops_rules.h"
// Reads count most, prints the number of parts; fails where they leave a gap, overlap or do not end.
int main() {
  long long count, most;
  while (scanf("%lld %lld", &count, &most) == 2) {
    long long at = 0, parts = 0;
    sf::in_parts(count, most, [&](int64_t first, int64_t n) {
      ++parts;
      if (first != at || n < 1 || n > most || parts > (count + most - 1) / most) {
        printf("%lld by %lld: part %lld from %lld, %lld\n", count, most, parts, (long long)first, (long long)n);
        exit(1);
      }
      at += n;
    });
    if (at != count) return 2;
    printf("%lld\n", parts);
  }
}
"""


def test_parts_of_a_count_cover_it_once(tmp_path_factory):
    """Up to the largest count of samples that a call takes, which the first one past the last part exceeds."""
    counts = (0, 1, 2, 4095, 4096, 4097, (1 << 31) - (1 << 21), (1 << 31) - (1 << 21) + 1, (1 << 31) - 1)
    calls = [(c, m) for c in counts for m in (1 << 10, (1 << 21) // 3, 1 << 21)]
    r = subprocess.run([_compiled(tmp_path_factory, "parts", PARTS)], input="".join("%d %d\n" % c for c in calls), capture_output=True,
                       text=True, timeout=60)
    assert r.returncode == 0, r.stdout
    assert [int(v) for v in r.stdout.split()] == [-(-c // m) for c, m in calls]


SPANS = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads samples tokens step groups, walks the workgroups of a sample as the kernel does and fails where rows are missed, taken
// twice or read past the sample. A wavefront's rows are walked at its first and its last three.
int main() {
  long long samples, tokens, groups;
  int step;
  while (scanf("%lld %lld %d %lld", &samples, &tokens, &step, &groups) == 4) {
    const sf::NormSpans p = sf::norm_spans(samples, tokens, step, groups);
    bool ok = p.span >= 1 && p.span % step == 0 && p.spans >= 1 && p.most >= 1 && (p.spans == 1 || p.spans * p.most <= 1 << 21);
    ok = ok && (long long)(p.spans - 1) * p.span < tokens && (long long)p.spans * p.span >= tokens;
    for (uint32_t b = 0; ok && b < p.spans; ++b) {
      const int start = (int)b * p.span, end = sf::span_end(start, p.span, (int)tokens);
      const long long want = (long long)(b + 1) * p.span;
      ok = end == (want < tokens ? want : tokens);
      for (int w = 0; ok && w < step && w < end - start; ++w) {
        const long long last = start + w + ((long long)end - 1 - start - w) / step * step;
        int token = start + w;
        ok = sf::row_ahead(token, step, end) == (token + (long long)step < end ? token + (long long)step : end - 1);
        if (last - 3ll * step > token) token = (int)(last - 3ll * step);
        for (;; token += step) {
          const int ahead = sf::row_ahead(token, step, end);
          ok = ok && token <= last && ahead >= start && ahead < end;
          if (!(ok && step < end - token)) break;
          ok = ahead == token + step;
        }
        ok = ok && token == last;
      }
    }
    if (!ok) {
      printf("%lld x %lld, %d rows at once, %lld groups: span %d, %u spans\n", samples, tokens, step, groups, p.span, p.spans);
      return 1;
    }
  }
}
"""


def test_workgroups_cover_a_samples_rows(tmp_path_factory):
    """Up to the largest count of tokens that a call takes, where the first row past the last workgroup's is 2^31."""
    top = (1 << 31) - 1
    counts = (1, 2, 3, 4, 5, 1001, 2048, 16384, 1 << 21, (1 << 21) + 1, (1 << 30) + 5, top - (1 << 21), top - (1 << 21) + 1, top - 4, top - 3,
              top - 1, top)
    calls = [(s, t, step, g) for t in counts for s in sorted({1, 2, 3, 1000, top // t}) if s * t <= top for step in (1, 4)
             for g in (512, 768, 1024)]
    r = subprocess.run([_compiled(tmp_path_factory, "spans", SPANS)], input="".join("%d %d %d %d\n" % c for c in calls),
                       capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


TILES = r"""
#include <cstdio>
#include "sf_ops_rules.h"
// Reads rows D, prints the pieces and wavefronts of a row, and whether that holds it and has a kernel.
int main() {
  long long rows;
  int D;
  while (scanf("%lld %d", &rows, &D) == 2) {
    const sf::NormTile t = sf::choose_norm_tile(rows, D);
    printf("%d %d %d\n", t.pieces, t.waves, (int)(256 * t.pieces * t.waves >= D && sf::norm_has_tile(t, D % 4 == 0)));
  }
}
"""


def _tiles(tmp_path_factory, calls):
    out = subprocess.run([_compiled(tmp_path_factory, "tiles", TILES)], input="".join("%d %d\n" % c for c in calls), capture_output=True,
                         text=True, check=True, timeout=60).stdout.split()
    out = [int(v) for v in out]
    return list(zip(out[::3], out[1::3], (d % 4 == 0 for _, d in calls))), out[2::3]


def test_a_row_fits_what_takes_it(tmp_path_factory):
    calls = [(rows, d) for d in range(1, 16385) for rows in (1, 2047, 2048, 1 << 20)]
    tiles, fit = _tiles(tmp_path_factory, calls)
    assert len(fit) == len(calls) and all(fit)
    kernels = open(os.path.join(CSRC, "k_residual_norm.hip")).read()
    named = {(int(p), int(w)) for p, w in re.findall(r"X\((\d+), (\d+)\)", kernels)}
    assert named == {t[:2] for t in tiles}


def test_the_gpu_tests_reach_every_kernel_of_the_norms(tmp_path_factory):
    tree = ast.parse(open(os.path.join(ROOT, "tests", "test_gpu_norm_tiles.py")).read())
    few, many = (next(ast.literal_eval(n.value) for n in tree.body if isinstance(n, ast.Assign) and n.targets[0].id == name)
                 for name in ("FEW", "MANY"))
    every = set(_tiles(tmp_path_factory, [(rows, d) for d in range(1, 16385) for rows in (1, 2048)])[0])
    assert all(s * t < 2048 for s, t, _ in few) and all(s * t >= 2048 for s, t, _ in many)
    assert set(_tiles(tmp_path_factory, [(s * t, d) for s, t, d in few + many])[0]) == every
    only_many = every - set(_tiles(tmp_path_factory, [(1, d) for d in range(1, 16385)])[0])
    assert only_many == {(3, 1, True), (4, 1, True), (5, 1, True)}
