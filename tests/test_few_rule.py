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


SPLIT = r"""
#include <cstdio>
#include "qlin_tiles.h"
int main() {
  int kind, sms; long long m, n, k;
  while (std::scanf("%d %lld %lld %lld %d", &kind, &m, &n, &k, &sms) == 5)
    std::printf("%d %d\n", qlin::choose_split_k((qlin::GemmKind)kind, m, n, k, sms),
                (int)qlin::split_over_few((qlin::GemmKind)kind, m, n, k, sms));
}
"""


def test_split_rule(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "split.cpp").write_text(SPLIT)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-I" + csrc, str(tmp_path / "split.cpp"), "-o", str(tmp_path / "split")],
                   check=True)

    def rule(kind, m, n, k):
        out = subprocess.run([str(tmp_path / "split")], input="%d %d %d %d 152\n" % (kind, m, n, k), capture_output=True,
                             text=True, check=True).stdout.split()
        return int(out[0]), int(out[1])

    nvfp4, fp8, f16 = 0, 1, 2
    assert rule(nvfp4, 552, 832, 4096)[0] == 4 and rule(nvfp4, 552, 832, 3840)[0] == 1     # 16 stages, 15
    assert rule(fp8, 552, 832, 4096)[0] == 4 and rule(fp8, 552, 832, 3968)[0] == 1
    assert rule(f16, 552, 832, 1280)[0] == 4 and rule(f16, 552, 832, 1216)[0] == 1
    assert rule(f16, 300, 3072, 1472)[0] == 1 and rule(f16, 300, 3072, 1536)[0] == 2       # 72 tiles
    assert rule(f16, 300, 3328, 12288)[0] == 1                                             # 78
    assert rule(f16, 352, 640, 4096)[0] == 8 and rule(f16, 512, 512, 4096)[0] == 4         # 15 tiles, 16
    assert rule(f16, 2**31 - 1, 2**40, 12288)[0] == 1
    # against the few-token kernel: more than 64 tokens, much of W to read
    assert rule(f16, 552, 64, 4096)[1] == 0 and rule(f16, 176, 768, 2560)[1] == 1
    assert rule(f16, 64, 768, 12288)[1] == 0 and rule(f16, 65, 768, 12288)[1] == 1
    assert rule(nvfp4, 552, 128, 4096)[1] == 0 and rule(nvfp4, 352, 128, 12288)[1] == 1
    # every split leaves each CTA a stage
    for kind in (nvfp4, fp8, f16):
        for m in (17, 129, 500, 2000):
            for n in (64, 320, 1024, 3072):
                for k in range(64, 6145, 320):
                    s = rule(kind, m, n, k)[0]
                    row = k // 2 if kind == nvfp4 else 2 * k if kind == f16 else k
                    assert s == 1 or s <= (row + 127) // 128


WIDE = r"""
#include <cstdio>
#include "qlin_tiles.h"
int main() {
  int kind, epi; long long m, n, k;
  while (std::scanf("%d %d %lld %lld %lld", &kind, &epi, &m, &n, &k) == 5)
    std::printf("%d\n", (int)qlin::choose_tile((qlin::GemmKind)kind, (qlin::Epilogue)epi, m, n, k, 152));
}
"""


def test_wide_tiles(tmp_path):
    # 128 x 192 for 16-bit linears alone, where they save a wave
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "wide.cpp").write_text(WIDE)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-I" + csrc, str(tmp_path / "wide.cpp"), "-o", str(tmp_path / "wide")], check=True)
    f16, linear = 2, 3
    cases = [((f16, linear, 1333, 2112, 1088), 3), ((f16, linear, 1333, 2112, 256), 3),
             ((f16, linear, 2000, 5120, 1088), 3), ((f16, linear, 2048, 2048, 1088), 1),
             ((f16, linear, 512, 3072, 1088), 1), ((f16, linear, 4608, 12288, 3072), 0)]
    every = [(kind, epi, m, n, k) for kind in (0, 1, 2) for epi in (0, 1, 2, 3, 4) if (kind, epi) != (f16, linear)
             for m, n in ((1333, 2112), (2000, 5120), (4608, 1024)) for k in (256, 1088, 3072)]
    text = "".join("%d %d %d %d %d\n" % c for c in [c for c, _ in cases] + every)
    out = [int(v) for v in subprocess.run([str(tmp_path / "wide")], input=text, capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert out[:len(cases)] == [w for _, w in cases] and 3 not in out[len(cases):]
