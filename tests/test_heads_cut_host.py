"""How rows and heads are shared out, on the CPU: all of them, once, for the GPU that there is."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "lq_heads_cut.h"
extern "C" void cut(int rows, int h0, int h1, int groups, int sms, int* out) {
  const LqHeadsCut c = lq_heads_cut(rows, h0, h1, groups, sms);
  const int v[] = {c.walk, c.parts[0], c.parts[1], c.block_rows, c.blocks, c.blocks_y};
  for (int i = 0; i < 6; ++i) out[i] = v[i];
}
"""
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    (d / "cut.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_18117_b200", "csrc"),
                    str(d / "cut.cpp"), "-o", str(d / "cut.so")], check=True)
    lib = C.CDLL(str(d / "cut.so"))

    def get(*a):
        out = (C.c_int * 6)()
        lib.cut(*a, out)
        return tuple(out)

    return get


@pytest.mark.parametrize("sms", [148, 132, 74, 16])
@pytest.mark.parametrize("groups", [1, 2, 3, 4, 8, 32])
def test_every_row_and_head_has_a_warp(cut, sms, groups):
    fill = 24 * sms
    for rows in (1, 2, 3, 31, 455, 887, 888, 889, 1775, 1776, 4096, 32760, 1 << 20, MOST - 1, MOST):
        for h0, h1 in ((1, 0), (0, 3), (16, 16), (32, 8), (20, 5), (28, 4), (64, 1), (4095, 7), (4096, 4096)):
            walk, p0, p1, block_rows, blocks, blocks_y = cut(rows, h0, h1, groups, sms)
            assert walk % groups == 0 and walk > 0
            for h, p in ((h0, p0), (h1, p1)):
                assert p * walk >= h and (p - 1) * walk < max(h, 1)
            assert 1 <= block_rows <= 2 and (blocks - 1) * block_rows < rows <= blocks * block_rows
            assert 1 <= blocks_y <= 65535 and block_rows * (p0 + p1) <= 1 << 14        # the kernel's quotients
            # longer walks than one step only where the rows' parts fill the GPU that there is
            assert walk == groups or rows * (p0 + p1) >= fill


def test_a_smaller_gpu_is_filled_by_fewer_rows(cut):
    assert cut(888, 16, 16, 3, 148)[0] == 15 and cut(888, 16, 16, 3, 74)[0] == 18
    assert cut(1000, 16, 16, 3, 148)[3] == 1 and cut(1000, 16, 16, 3, 74)[3] == 2


def test_the_cuts_of_the_sizes_that_were_timed(cut):
    assert cut(1, 16, 16, 3, 148) == (3, 6, 6, 1, 1, 3)
    assert cut(8192, 16, 16, 3, 148) == (18, 1, 1, 2, 4096, 1)
    assert cut(32760, 20, 20, 4, 148) == (20, 1, 1, 2, 16380, 1)
    assert cut(4100, 28, 4, 2, 148) == (8, 4, 1, 2, 2050, 1)
