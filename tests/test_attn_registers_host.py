"""Registers of the attention's tile kernel, as ptxas reports them: the split among its warps takes no more than every instance is launched with."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2604_18117_b200", "csrc", "lq_attn_tile.cu")


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="nvcc not found")
def test_every_instance_is_launched_with_the_registers_that_its_warps_share(tmp_path):
    r = subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.dirname(SOURCE), "-c", SOURCE, "-o", str(tmp_path / "a.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    used = re.findall(r"Compiling entry function '\S*lq_attn_tile_kernel\S*' for[^\n]*\n(?:(?!Compiling)[^\n]*\n)*?[^\n]*Used (\d+) registers", r.stderr)
    with open(SOURCE) as f:
        source = f.read()
    soft, opening = map(int, re.search(r"SOFT_WARPS = (\d+), OPEN_WARPS = (\d+)", source).groups())
    launch, most, lean = map(int, re.search(r"LAUNCH_REGS = (\d+), SOFT_REGS = (\d+), LEAN_REGS = (\d+);", source).groups())
    warps = soft + opening + 1
    assert len(used) == 5 and warps % 4 == 0
    assert all(soft * most + (warps - soft) * lean <= warps * int(n) and int(n) == launch for n in used), used
