"""The staging boxes of a warp's TMA stores (csrc/qlin_tiles.h, host code): a store may
not take the box of the store just before it, in whatever numbers a tile's stores come
and from tile to tile.  Also the sizes of test_gpu_staged_stores.py: they have to take
the tiles with odd numbers of stores, more of them than a GPU has SMs."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

SMS = 152
F16, FP8, NVFP4 = 2, 1, 0
PLAIN, LINEAR = 0, 3
NARROW, WIDE = 2, 3
WIDTH = {NARROW: 64, WIDE: 192}
# M, N, K.  N % 192 is 0, 64 and 128: a last tile of all, two and four of its six chunks of 32
WIDE_SIZES = [(2000, 5120, 64), (2000, 5120, 192), (448, 9792, 128), (2000, 2752, 64), (1300, 3648, 192)]
NARROW_SIZES = [(320, 6464, 64), (257, 6464, 128)]

MAIN = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include "qlin_tiles.h"
int main(int argc, char**) {
  if (argc > 1) {
    qlin::StagingBoxes boxes;
    int stores;   // of the next tile
    while (std::scanf("%d", &stores) == 1)
      for (int i = 0; i < stores; ++i) std::printf("%d\n", boxes.take());
    return 0;
  }
  int kind, epi, sms; long long m, n, k;
  while (std::scanf("%d %d %lld %lld %lld %d", &kind, &epi, &m, &n, &k, &sms) == 6)
    std::printf("%d\n", (int)qlin::choose_tile((qlin::GemmKind)kind, (qlin::Epilogue)epi, m, n, k, sms));
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("boxes")
    (d / "main.cpp").write_text(MAIN)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-I" + csrc, str(d / "main.cpp"), "-o", str(d / "main")], check=True)

    def call(text, *args):
        out = subprocess.run([str(d / "main"), *args], input=text, capture_output=True, text=True, check=True)
        return [int(v) for v in out.stdout.split()]
    return call


@pytest.mark.parametrize("tiles", [[1] * 9, [3] * 9, [2] * 9, [3, 3, 2, 1, 0, 3], [1, 0, 0, 1, 2, 1], [2, 1, 2, 3, 1]])
def test_no_store_takes_the_box_before_it(run, tiles):
    boxes = run(" ".join(map(str, tiles)), "boxes")
    assert len(boxes) == sum(tiles) and set(boxes) <= {0, 1}
    assert all(a != b for a, b in zip(boxes, boxes[1:]))


def test_sizes_take_several_tiles_with_odd_numbers_of_stores(run):
    cases = [(F16, LINEAR, s, WIDE) for s in WIDE_SIZES]
    cases += [(kind, epi, s, NARROW) for kind in (FP8, NVFP4) for epi in (PLAIN, LINEAR) for s in NARROW_SIZES]
    got = run("".join("%d %d %d %d %d %d\n" % (kind, epi, *s, SMS) for kind, epi, s, _ in cases))
    assert got == [tile for _, _, _, tile in cases]
    for _, _, (M, N, _), tile in cases:
        assert -(-M // 128) * -(-N // WIDTH[tile]) > SMS
