"""Rows of a sequence, on the CPU: whatever the array of first rows holds, they stay within the call's."""
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_18117_b200", "csrc")
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def rows_of(tmp_path_factory):
    import ctypes as C
    d = tmp_path_factory.mktemp("rows")
    (d / "r.cpp").write_text('#include "lq_kv_rows.h"\nextern "C" void f(int a, int b, int rows, int* out) { const LqRowRange r = lq_kv_rows(a, b, rows); out[0] = r.row; out[1] = r.n; }\n')
    # (an overflow of signed numbers ends the program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    so, out = C.CDLL(str(d / "r.so")), (C.c_int * 2)()

    def f(a, b, rows):
        so.f(a, b, rows, out)
        return tuple(out)
    return f


def test_rows_stay_within_the_call(rows_of):
    ends = [LOW, LOW + 1, -7, -1, 0, 1, 2, 5, 9, 10, 11, HIGH - 1, HIGH]
    for a, b, rows in itertools.product(ends, ends, [0, 1, 10, HIGH]):
        first = min(max(a, 0), rows)
        assert rows_of(a, b, rows) == (first, max(0, min(b, rows) - first)), (a, b, rows)
