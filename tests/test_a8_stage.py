"""The loads of the 8-bit product's blocks (csrc/a8_stage.h), walked on the CPU: every lane of every phase, those behind K among them, reads the piece
that it should or is out of range, by the rule that a raw buffer load is in range where lane offset < bytes - scalar offset in unsigned arithmetic."""
import ctypes
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_13565_amd", "csrc")

WALK = r"""
#include "a8_stage.h"
using namespace mxfp4::a8;
// Of an operand whose step is step_bytes of a row of row_bytes: `have` rows of a block of `rows`, phases of `s` steps, `ahead` of them behind the last.
// 0, or which check fails first.
extern "C" int walk(int rows, int have, int row_bytes, int steps, int step_bytes, int s, int ahead, int* phase)
{
    const int chunks = s * step_bytes / 16;
    const unsigned bytes = (unsigned)(have * row_bytes);
    for (int p = 0; p < (steps + s - 1) / s + ahead; ++p) {
        *phase = p;
        const int from = phase_from(p * s, steps, step_bytes), first = phase_chunk(p * s, step_bytes);
        if (from < 0 || (unsigned)from > bytes)
            return 1;
        for (int piece = 0; piece < rows * chunks; ++piece) {
            const int row = piece_row(piece, chunks), chunk = p * s * (step_bytes / 16) + piece_chunk(piece, chunks);
            const unsigned lane = (unsigned)(piece_offset(piece, chunks, have, row_bytes) | past(row_bytes / 16 - 1, first + piece_chunk(piece, chunks)));
            const bool live = row < have && chunk * 16 < row_bytes, in_range = lane < bytes - (unsigned)from;
            if (live != in_range)
                return 2;
            if (live && lane + (unsigned)from != (unsigned)(row * row_bytes + chunk * 16))
                return 3;
        }
    }
    return 0;
}
"""


def shapes():
    """(rows of x, weight rows, steps a phase, phases ahead) of the blocks that the two files launch."""
    found = set()
    text = open(os.path.join(CSRC, "gemm_a8_mid.hip")).read()
    for wm, wn, wk, mf, nf, d in re.findall(r"launch<(\d+), (\d+), (\d+), (\d+), (\d+), (\d+)>\(a", text):
        found.add((int(wm) * int(mf) * 32, int(wn) * int(nf) * 32, int(wk), int(d)))
    text = open(os.path.join(CSRC, "gemm_a8.hip")).read()
    for wn, wk, nf, rows, d in re.findall(r"launch<\d+, (\d+), (\d+), \d+, (\d+), (\d+), (\d+)>\(a", text):
        found.add((int(rows), int(wn) * int(nf) * 16, int(wk), int(d)))
    return sorted(found)


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("a8_stage")
    (d / "walk.cpp").write_text(WALK)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "walk.cpp"), "-o", str(d / "walk.so")])
    return ctypes.CDLL(str(d / "walk.so")).walk


def test_every_shape_is_known():
    assert len(shapes()) == 11


@pytest.mark.parametrize("m,n,s,ahead", shapes())
def test_loads_are_of_their_piece_or_out_of_range(walk, m, n, s, ahead):
    phase = ctypes.c_int()
    for k in (32, 64, 96, 128, 160, 416, 128 * s - 32, 128 * s, 128 * s + 32, 1376, 4096):
        steps = (k + 127) // 128
        for rows, row_bytes, step_bytes in ((m, k, 128), (n, k // 2, 64)):
            for have in sorted({min(h, rows) for h in (1, 2, 3, 4, 5, rows - 1, rows)} - {0}):
                failed = walk(rows, have, row_bytes, steps, step_bytes, s, ahead, ctypes.byref(phase))
                assert failed == 0, "check %d: phase %d of K = %d, %d of %d rows" % (failed, phase.value, k, have, rows)
