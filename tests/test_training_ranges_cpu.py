"""Which words the training kernels read around rows that start on any byte, by the functions the kernels call
(csrc/pg_train_ranges.h), compiled for the host and run over widths, tiles and alignments."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2008_01425_b200", "csrc")
SOURCE = r"""
#include "pg_train_ranges.h"
extern "C" int scales(int cols, int col) { return pgt::scales_of_tile(cols, col); }
extern "C" int words(unsigned long long from, int count) { return pgt::words_of_scales(static_cast<uintptr_t>(from), count); }
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    d = tmp_path_factory.mktemp("ranges")
    src, lib = str(d / "ranges.cpp"), str(d / "ranges.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-o", lib, src])
    L = ctypes.CDLL(lib)
    L.words.argtypes = [ctypes.c_ulonglong, ctypes.c_int]
    return L


@pytest.mark.parametrize("blocks", [1, 2])
def test_every_word_of_scales_holds_one_of_the_row(ranges, blocks):
    """The 8-bit weight gradient's tiles of 128 rows of A (features), by single blocks and in pairs: every word that is
    read holds a scale of the row it is read for, and every scale that a tile needs is in a word that is read."""
    for cols in range(1, 1300):
        have = -(-cols // 32)
        for m0 in range(0, -(-cols // (128 * blocks)) * 128 * blocks, 128):
            count = ranges.scales(cols, m0)
            assert count == max(0, min(4, have - m0 // 32))
            for row in range(4):                      # the row's first scale, at each place of a word
                at = row + m0 // 32
                words = ranges.words(at, count)
                read = [range((at & ~3) + 4 * w, (at & ~3) + 4 * w + 4) for w in range(words)]
                of_row = range(row, row + have)
                assert all(any(b in of_row for b in r) for r in read), (cols, m0, row)
                assert all(any(b in r for r in read) for b in range(at, at + count)), (cols, m0, row)
