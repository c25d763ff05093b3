"""Items of the few-row attention that meet in a CTA: the last CTA of one, alone in its group of those
that join their sums, begins the next, whose count it shares a place with.  Where that happens follows
from the split of the work, which is run here as the kernel runs it (csrc/qlin_cache.h), for every
number of CTAs that the grid may have."""
import math
import os
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")

from conftest import ROOT
from test_gpu_cache import FORMATS, _check, _fill, _gen, _make

from paper_2609_21849_gb300 import qlin

# For two sequences of one new token and KV head: keys of the first and of the second such that they meet
# like that in some CTA, both with several CTAs.
MAIN = r"""
#include <cstdio>
#include "qlin_cache.h"
using namespace qlin;
int main() {
  int bytes, rows_max, rows, head_dim, ctas;
  while (std::scanf("%d %d %d %d %d", &bytes, &rows_max, &rows, &head_dim, &ctas) == 5) {
    const int tile = kFewWarps * few_warp_keys(bytes, rows_max), least = few_least(tile);
    const int group = few_join_group(rows, head_dim);
    long long found_a = 0, found_b = 0;
    // (every CTA with work, and runs of few tiles)
    for (long long total = (long long)least * ctas; total < (long long)(least + 3) * ctas && !found_a; total += 7)
      for (long long a = 1 + kFewItemCost; a < total - kFewItemCost && !found_a; ++a) {
        const long long working = split_ctas(total, ctas, least);
        const Split s = split_evenly(total, working);
        const long long last_a = split_owner(s, a - kFewItemCost - 1), first_b = split_owner(s, a),
                        last_b = split_owner(s, total - kFewItemCost - 1), first_a = split_owner(s, 0);
        if (last_a == first_b && last_a > first_a && last_b > first_b && (last_a - first_a) % group == 0) {
          found_a = (a - kFewItemCost) * tile;
          found_b = (total - a - kFewItemCost) * tile;
        }
      }
    std::printf("%lld %lld\n", found_a, found_b);
  }
}
"""

SHAPES = [(64, 1, 16), (64, 16, 16), (256, 16, 16), (64, 24, 32)]   # head_dim, rows, rows of an MMA


def _places(tmp_path, lines):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2609_21849_gb300", "csrc"),
                    str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    out = subprocess.run([str(tmp_path / "main")], input="\n".join(lines), capture_output=True, text=True, check=True)
    return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]


def _grids(sms, bytes_, D, rows, most):
    return [f"{bytes_} {most} {rows} {D} {per * sms}" for per in (1, 2, 3, 4)]


@pytest.mark.parametrize("sms", [148, 152, 160])
@pytest.mark.parametrize("bytes_", [1, 2])
def test_such_lengths_exist(sms, bytes_, tmp_path):
    lines = [g for D, rows, most in SHAPES for g in _grids(sms, bytes_, D, rows, most)]
    for line, (a, b) in zip(lines, _places(tmp_path, lines), strict=True):
        assert a > 0 and b > 0, line


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("D,G,most", SHAPES)
def test_items_that_meet(D, G, most, fmt, dtype, tmp_path):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    ws = qlin.alloc_cache_attention_workspace()
    for a, b in _places(tmp_path, _grids(sms, 1 if fmt == "e4m3" else 2, D, G, most)):
        assert a > 0 and b > 0
        cached = [a - 1, b - 1]
        # (pages of 24 slots keep more than 16 rows with this kernel)
        c = _make(cached, [1, 1], 1, D, 24 if G > 16 else 64, fmt, a)
        _fill(c, cached, [1, 1], a + 1)
        q = torch.randn(2, G, D, generator=_gen(a + 2), device="cuda").to(dtype)
        first = qlin.qlin_cache_attention(c, q, 1 / math.sqrt(D), workspace=ws)
        assert not ws[:8192].any()
        _check(c, q, 1 / math.sqrt(D), None, fmt, first, None)
        for _ in range(5):
            assert torch.equal(qlin.qlin_cache_attention(c, q, 1 / math.sqrt(D), workspace=ws), first)
        assert not ws[:8192].any()
        assert qlin.qlin_sync_status() == 0
