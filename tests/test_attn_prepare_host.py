"""A cache is refused where the attention's tile kernel was built with fewer registers than its warps share: it would wait for them for ever.  The library's own
check, with the runtime's answer about the kernel put in its place; nothing runs on a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_18117_b200", "csrc")
SOURCE = r"""
#include <stdio.h>
#include <stdlib.h>
#include "lq_kvcache.h"
static int regs, asked, set;
static cudaError_t answer;
cudaError_t lq_note_cuda(cudaError_t e) { return e; }
extern "C" cudaError_t __wrap_cudaFuncGetAttributes(cudaFuncAttributes* at, const void*) { ++asked; *at = cudaFuncAttributes(); at->numRegs = regs; return answer; }
extern "C" cudaError_t __wrap_cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { ++set; return cudaSuccess; }
int g_lq_overlap;
int main(int argc, char** argv) {
  lq_kvcache c = {};
  c.Dp = atoi(argv[1]); regs = atoi(argv[2]); answer = atoi(argv[3]) ? cudaErrorInvalidDeviceFunction : cudaSuccess;
  const int s = lq_attn_tile_prepare(&c);
  printf("%d %d %d\n", s, asked, set);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("nvcc") is None:
        pytest.skip("nvcc not found")
    d = tmp_path_factory.mktemp("prepare")
    (d / "main.cu").write_text(SOURCE)
    subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-cudart", "static", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    "-Xlinker", "--wrap=cudaFuncGetAttributes", "-Xlinker", "--wrap=cudaFuncSetAttribute", str(d / "main.cu"), os.path.join(CSRC, "lq_attn_tile.cu"),
                    "-o", str(d / "p")], check=True)
    return lambda *a: tuple(map(int, subprocess.run([str(d / "p"), *map(str, a)], check=True, capture_output=True, text=True).stdout.split()))


@pytest.mark.parametrize("Dp", [64, 80, 96, 112, 128])
def test_registers_that_a_kernel_was_built_with(program, Dp):
    assert program(Dp, 128, 0) == (0, 1, 1)
    assert program(Dp, 127, 0) == (2, 1, 0)
    assert program(Dp, 128, 1) == (4, 1, 0)
