"""Host-side walk (no GPU) of the function by which the row kernels find a row's sequence and position: what tables_append leaves when it
refuses chunks, or when more rows were set aside than asked for, must not lead behind a context."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import plain_8bit as P
from paper_2509_16495_amd import build as BLD

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++ to compile the function for the host")

SOURCE = r"""
#include "query_rows.h"
extern "C" void rows_of(const int32_t* cu, const int32_t* lens, int num_seqs, int rows, int32_t* seq, int32_t* pos) {
    for (int i = 0; i < rows; ++i) {
        const auto r = shiftattn::query_row(cu, lens, num_seqs, i);
        seq[i] = r.seq, pos[i] = r.pos;
    }
}
"""


@pytest.fixture(scope="module")
def rows_of(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("rows"))
    src, lib = os.path.join(d, "rows.cpp"), os.path.join(d, "rows.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-shared", "-fPIC", "-I", BLD.CSRC, src, "-o", lib])
    f = ctypes.CDLL(lib).rows_of

    def call(cu, lens, rows):
        lens = np.ascontiguousarray(lens, np.int32)
        cu = None if cu is None else np.ascontiguousarray(cu, np.int32)
        seq, pos = np.empty(rows, np.int32), np.empty(rows, np.int32)
        at = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)
        f(at(cu), at(lens), len(lens) if cu is None else len(cu) - 1, rows, at(seq), at(pos))
        return seq, pos
    return call


@pytest.mark.parametrize("new,had,blocks,spare", [
    ([4, 40], [5, 20], 2, 0), ([40, 4], [20, 5], 1, 0), ([7, 90, 12], [0, 0, 3], 3, 0), ([50], [0], 1, 0), ([3, 0, 5], [1, 0, 30], 9, 6),
    ([0, 0], [4, 0], 9, 5), ([5, 5, 5], [0, 0, 0], 0, 0)])
def test_rows_of_refused_chunks_have_no_token(rows_of, new, had, blocks, spare):
    """Every row of a chunk that was taken is its own token; every other row is nobody's."""
    first = [-(-h // 16) for h in had]
    t = P.Tables(had, 8, np.arange(100, 100 + blocks), blocks)
    for s, n in enumerate(first):
        t.table[s, :n] = np.arange(10 * s, 10 * s + n)
    total = sum(new) + spare
    cu, slots, taken = t.append(new, len(new), total, total)
    seq, pos = rows_of(cu, t.lens, total)
    want = [(s, had[s] + i) for s in range(len(new)) for i in range(taken[s])]
    assert list(zip(seq[:len(want)], pos[:len(want)])) == want
    assert (seq[len(want):] == -1).all() and (pos[len(want):] == -1).all() and (slots[len(want):] == -1).all()
    assert all(p < t.lens[s] for s, p in zip(seq, pos) if s >= 0)


def test_decode_rows_are_their_sequence(rows_of):
    seq, pos = rows_of(None, [3, 0, 17, -2], 4)
    assert seq.tolist() == [0, 1, 2, 3] and pos.tolist() == [2, -1, 16, -3]
