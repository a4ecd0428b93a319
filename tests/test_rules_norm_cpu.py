"""How the rows around a block are shared out over launches and workgroups, compiled for the host from the header that the
kernels include."""
import subprocess

from test_rules_cpu import _compiled

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
