"""How the verification of drafted tokens divides its rows among CTAs (csrc/draft_grid.h), on the CPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2412_07017_b200 import build as lib_build

PROBE = """
#include "draft_grid.h"
extern "C" int slices(int batch, int pieces, int fit, int pairs) { return asynclm::draft_slices(batch, pieces, fit, pairs != 0); }
"""
PAIRS, ALONE = 13 * 148, 18 * 148      # CTAs that fit


@pytest.fixture(scope="module")
def slices(tmp_path_factory):
    d = tmp_path_factory.mktemp("draft_grid")
    src, lib = os.path.join(d, "probe.cpp"), os.path.join(d, "probe.so")
    with open(src, "w") as f:
        f.write(PROBE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", lib_build.CSRC, "-o", lib, src], check=True)
    return ctypes.CDLL(lib).slices


# where another choice was measured to be slower
@pytest.mark.parametrize("batch,pairs,want", [(100, 1, 9), (150, 1, 6), (200, 1, 4), (237, 1, 4), (300, 1, 3), (355, 1, 2), (356, 1, 2), (473, 1, 2), (500, 1, 2), (700, 1, 2), (888, 1, 1),
                                              (128, 0, 10), (200, 0, 6), (300, 0, 4), (454, 0, 2), (545, 0, 2), (700, 0, 1), (907, 0, 1)])
def test_measured(slices, batch, pairs, want):
    assert slices(batch, 1 << 20, PAIRS if pairs else ALONE, pairs) == want


@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("fit", [PAIRS, ALONE, 13 * 132, 2, 1])
def test_no_batch_leaves_the_gpu_empty(slices, fit, pairs):
    """Of the half of the CTAs that fit, two thirds or more are used where rows are divided at all; a row is not left to one CTA while two of each fit that half;
    more sequences have no more CTAs each; 65 535 sequences have one."""
    last = 1 << 30
    for batch in range(1, 4000):
        s = slices(batch, 1 << 20, fit, pairs)
        assert 1 <= s <= last
        last = s
        if batch <= fit // 2:
            assert 3 * s * batch >= 2 * (fit // 2) or s == 1
            assert s > 1 or 2 * batch > fit // 2
            assert s * batch <= max(fit // 2, fit * 3 // 4 if s == 2 else 0)
        if pairs and 8 * batch <= 3 * fit - 8:
            assert s >= 2
    assert slices(65535, 1 << 20, fit, pairs) == 1


def test_no_more_ctas_than_pieces_for_their_warps(slices):
    for pieces in range(1, 40):
        for batch in (1, 3, 50):
            assert slices(batch, pieces, PAIRS, 1) <= (pieces + 1) // 2
