"""The paged cache's index arithmetic and the attention's split of its work
(csrc/qlin_cache.h, host and device code), compiled and run on the CPU."""
import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

MAIN = r"""
#include <cstdio>
#include <cstring>
#include "qlin_cache.h"
using namespace qlin;
int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    if (!std::strcmp(what, "place")) {
      long long at; int ps, w, i = -1, s = -1;
      std::scanf("%lld %d %d", &at, &ps, &w);
      const bool ok = cache_place(at, ps, w, &i, &s);
      std::printf("%d %d %d\n", (int)ok, ok ? i : -1, ok ? s : -1);
    } else if (!std::strcmp(what, "seq")) {
      long long a, b, c, t; int ps, w;
      std::scanf("%lld %lld %lld %lld %d %d", &a, &b, &c, &t, &ps, &w);
      const CacheSeq s = cache_seq(a, b, c, t, ps, w);
      std::printf("%d %d %lld\n", (int)s.bad, s.fresh, (long long)s.keys);
    } else {
      long long total, ctas, least;
      std::scanf("%lld %lld %lld", &total, &ctas, &least);
      const long long n = split_ctas(total, ctas, least);
      const Split s = split_evenly(total, n);
      std::printf("%lld", n);
      for (long long c = 0; c <= n; ++c) std::printf(" %lld", (long long)split_begin(s, c));
      for (long long t = 0; t < total; t += total / 997 + 1) std::printf(" %lld", (long long)split_owner(s, t));
      std::printf("\n");
    }
  }
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("cache")
    (d / "main.cpp").write_text(MAIN)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I" + csrc,
                    str(d / "main.cpp"), "-o", str(d / "main")], check=True)

    def go(lines):
        out = subprocess.run([str(d / "main")], input="\n".join(lines), capture_output=True, text=True, check=True)
        return [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
    return go


def test_places(run):
    cases = [(0, 8, 1), (7, 8, 1), (8, 8, 1), (8, 8, 2), (-1, 8, 2), (2**31 + 5, 16, 2**28), (2**40, 256, 2**31 - 1),
             (100, 7, 15), (104, 7, 15), (105, 7, 15)]
    got = run([f"place {a} {p} {w}" for a, p, w in cases])
    for (at, p, w), g in zip(cases, got):
        inside = 0 <= at < p * w
        assert g == ([1, at // p, at % p] if inside else [0, -1, -1]), (at, p, w)


def test_sequences(run):
    # (start, end, cached, tokens, page size, table width) -> (bad, new tokens, keys)
    cases = {(0, 5, 10, 5, 8, 2): (0, 5, 15), (0, 5, 11, 5, 8, 2): (0, 5, 16), (0, 5, 12, 5, 8, 2): (1, 5, 16),
             (3, 3, 40, 9, 8, 2): (0, 0, 16), (4, 3, 0, 9, 8, 2): (1, 0, 0), (-1, 3, 0, 9, 8, 2): (1, 0, 0),
             (0, 10, 0, 9, 8, 2): (1, 0, 0), (0, 1, -1, 9, 8, 2): (1, 0, 0),
             (0, 1, 2**31 - 1, 1, 256, 2**24): (0, 1, 2**31)}
    got = run(["seq %d %d %d %d %d %d" % c for c in cases])
    assert got == [list(v) for v in cases.values()]


def test_every_unit_has_one_owner(run):
    rng = random.Random(0)
    cases = [(1, 1, 1), (1, 600, 4), (599, 600, 1), (600, 600, 1), (601, 600, 1), (2**42, 1024, 1)]
    cases += [(rng.randint(1, 10**rng.randint(1, 12)), rng.randint(1, 1024), rng.randint(1, 8)) for _ in range(300)]
    for (total, ctas, least), g in zip(cases, run([f"split {t} {c} {n}" for t, c, n in cases])):
        n, begins, owners = g[0], g[1:g[0] + 2], g[g[0] + 2:]
        assert 1 <= n <= ctas and begins[0] == 0 and begins[-1] == total
        sizes = [b - a for a, b in zip(begins, begins[1:])]
        assert max(sizes) - min(sizes) <= 1
        if total >= n * least:
            assert min(sizes) >= least - 1
        for t, o in zip(range(0, total, total // 997 + 1), owners):
            assert begins[o] <= t < begins[o + 1]
