"""The rule that sends a linear to the few-token kernel (csrc/qlin_tiles.h, host code),
compiled and run on the CPU."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

MAIN = r"""
#include <cstdio>
#include "qlin_tiles.h"
int main() {
  int f16, sms; long long m, n, row;
  while (std::scanf("%d %lld %lld %lld %d", &f16, &m, &n, &row, &sms) == 5)
    std::printf("%d\n", (int)qlin::few_tokens(f16 != 0, m, n, row, sms));
}
"""


def test_rule(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "main.cpp").write_text(MAIN)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-I" + csrc, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")],
                   check=True)
    # (16-bit operands, M, N, bytes of W's rows) -> few
    cases = [((0, 1, 64, 32), 1), ((0, 16, 1 << 20, 6144), 1),          # always up to 16 tokens
             ((0, 17, 3072, 1536), 1), ((0, 32, 3136, 1536), 1),        # 2.6 units per SM: 395 of 152
             ((0, 32, 3200, 1536), 0), ((0, 33, 3072, 3072), 0),
             ((1, 32, 6144, 6144), 1), ((1, 33, 6144, 6144), 0),        # 16-bit operands: 5.2
             ((1, 128, 64, 128), 1), ((1, 3152, 64, 128), 1), ((1, 3153, 64, 128), 0),
             ((0, 1568, 64, 2048), 1), ((0, 1585, 64, 2048), 0),
             ((0, 1152, 64, 2047), 1), ((0, 1153, 64, 2047), 0),        # 1.9 over short rows: 288
             ((0, 2**31 - 1, 64, 2048), 0), ((0, 17, 2**40, 2048), 0)]
    text = "".join("%d %d %d %d 152\n" % c for c, _ in cases)
    out = subprocess.run([str(tmp_path / "main")], input=text, capture_output=True, text=True, check=True)
    assert [int(v) for v in out.stdout.split()] == [w for _, w in cases]
