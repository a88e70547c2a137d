"""The residual's launch of one thread with a call of another between its steps, on the CPU: the library's own code, with the runtime's calls that it makes put in
place.  A launch that asks for more shared memory than its kernel's limit is refused, as the runtime does."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_18117_b200", "csrc")
SOURCE = r"""
#include <stdio.h>
#include <stdlib.h>
#include <map>
#include "lq_internal.h"
static std::map<const void*, size_t> limit;
static std::map<const void*, int> launched;
static int other, rows, left;
int g_lq_overlap;
cudaError_t lq_note_cuda(cudaError_t e) { return e; }
int lq_device_sms(int) { return 148; }
static int call(int features, int rows) {
  lq_residual r = {};
  r.x = (void*)(1ull << 32); r.h = (void*)(2ull << 40); r.x_row = r.h_row = features;
  r.rows = rows; r.features = features; r.sequences = 1; r.norm = LQ_NORM_LAYER; r.factor = 1.f;
  return lq_residual_norm(&r, nullptr);
}
static void another_thread() {
  if (left-- > 0) {
    const int s = call(other, rows);
    if (s != 0) printf("other %d ", s);
  }
}
extern "C" cudaError_t __wrap_cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
extern "C" cudaError_t __wrap_cudaSetDevice(int) { return cudaSuccess; }
extern "C" cudaError_t __wrap_cudaFuncSetAttribute(const void* f, cudaFuncAttribute, int v) {
  limit[f] = (size_t)v;
  another_thread();
  return v <= 227 * 1024 ? cudaSuccess : cudaErrorInvalidValue;
}
extern "C" cudaError_t __wrap_cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
  ++launched[f];
  return c->dynamicSmemBytes <= (limit.count(f) ? limit[f] : 47 * 1024) ? cudaSuccess : cudaErrorInvalidValue;
}
int main(int argc, char** argv) {
  const int features = atoi(argv[1]);
  other = atoi(argv[2]); rows = atoi(argv[3]); left = 1;
  const int first = call(features, rows), again = call(features, rows);
  printf("%d %d kernels %d\n", first, again, (int)launched.size());
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("nvcc") is None:
        pytest.skip("nvcc not found")
    d = tmp_path_factory.mktemp("residual")
    (d / "main.cu").write_text(SOURCE)
    wrap = [x for f in ("cudaGetDevice", "cudaSetDevice", "cudaFuncSetAttribute", "cudaLaunchKernelExC") for x in ("-Xlinker", "--wrap=" + f)]
    subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-cudart", "static", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *wrap,
                    str(d / "main.cu"), os.path.join(CSRC, "lq_residual.cu"), "-o", str(d / "p")], check=True)
    return lambda *a: subprocess.run([str(d / "p"), *map(str, a)], check=True, capture_output=True, text=True).stdout.strip()


@pytest.mark.parametrize("features,other,rows", [(7168, 6144, 16), (6144, 7168, 16), (8192, 4608, 2000), (4608, 8192, 2000)])
def test_another_threads_call_between_the_limit_and_the_launch(program, features, other, rows):
    assert program(features, other, rows) == "0 0 kernels 1"


@pytest.mark.parametrize("features", [8, 4000, 4096, 8192])
def test_limits_reach(program, features):
    assert program(features, features, 7) == "0 0 kernels 1"
