"""What the cache's, the attention's and the residual's entry points refuse without a GPU, and their structures' layouts."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2604_18117_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _code(f, *a):
    with pytest.raises(B.LqError) as e:
        f(*a)
    return e.value.code


def test_sizes_of_a_cache():
    for bad in ((0, 1, 32, 1, 64), (1, 0, 32, 1, 64), (1, 1, 0, 1, 64), (1, 1, 32, 0, 64), (1, 1, 32, 1, 0), (-1, 1, 32, 1, 64)):
        assert _code(B.lq_kvcache_create, *bad) == 1, bad
    for bad in ((1, 1, 31, 1, 64), (1, 1, 65568, 1, 64), (1, 1, 32, 4097, 64), (1, 1, 32, 1, 68), (1, 1, 32, 1, 264)):
        assert _code(B.lq_kvcache_create, *bad) == 2, bad
    assert _code(B.lq_kvcache_create, 1000, 2 ** 30, 65536, 4096, 256) == 3           # more than any memory; no product leaves 64 bits


def test_null_handles_and_structures():
    L = B.lib()
    assert L.lq_kvcache_create(1, 1, 32, 1, 64, 0, None) == 1 and L.lq_kvcache_free(None) == 1
    batch, rows, attn = B.lq_kvbatch(1, 1, 4096, 4096, 1), B.lq_kvrows(4096, (0, 8, 8), 8192, (0, 8, 8)), B.lq_attn(4096, (8, 8), 8192, (8, 8), 1, 1.0)
    assert L.lq_kvcache_append(None, 0, batch, rows, 0, None) == 1 and L.lq_kvcache_read(None, 0, batch, None, 1, rows, 0, None) == 1
    assert L.lq_cache_attention(None, 0, batch, attn, None) == 1 and L.lq_cache_attention(None, 0, batch, None, None) == 1
    assert L.lq_residual_norm(None, None) == 1


def test_residual_arguments():
    make = lambda **k: B.lq_residual(**{**dict(rows=8, features=64, x_ptr=1 << 20, x_out_ptr=2 << 20, h_ptr=3 << 20, y_ptr=4 << 20), **k})
    for k in (dict(x_ptr=0), dict(x_out_ptr=0, h_ptr=0), dict(rows=0), dict(features=-8), dict(sequences=3), dict(after=3), dict(norm=-1), dict(h_dtype=2), dict(eps=-1.0),
              dict(factor=float("nan")), dict(y_ptr=0, after=1), dict(weight_ptr=16), dict(bias_ptr=16, norm=1), dict(x_ptr=(1 << 20) + 8), dict(strides=(60, 64, 64, 64)),
              dict(h_ptr=1 << 20), dict(x_out_ptr=4 << 20), dict(x_out_ptr=3 << 20), dict(h_ptr=4 << 20, h_dtype=1), dict(strides=(64, 64, 64, 32)),
              dict(gate_ptr=2 << 20), dict(norm=1, weight_ptr=3 << 20)):
        assert _code(B.lq_residual_norm, make(**k)) == 1, k
    for k in (dict(features=60), dict(features=8200), dict(strides=(64, 64, 1 << 40, 64))):
        assert _code(B.lq_residual_norm, make(**k)) == 2, k


def test_layouts_of_the_structures(tmp_path):
    """The header's, as a C compiler lays them out, field by field."""
    names = {"lq_kvbatch": B.LqKvBatch, "lq_kvrows": B.LqKvRows, "lq_attn": B.LqAttn, "lq_residual": B.LqResidual}
    lines = [f'printf("{n} size %zu\\n", sizeof({n}));' for n in names]
    lines += [f'printf("{n} {f} %zu\\n", offsetof({n}, {f}));' for n, c in names.items() for f, _ in c._fields_]
    src = tmp_path / "l.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "lq.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")], check=True)
    for line in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines():
        n, f, v = line.split()
        assert int(v) == (C.sizeof(names[n]) if f == "size" else getattr(names[n], f).offset), line


def test_structures_hold_what_they_are_given():
    get = lambda s: [getattr(s, f) for f, _ in s._fields_]
    for s, c in ((B._KV_BATCH, B.LqKvBatch), (B._KV_ROWS, B.LqKvRows), (B._ATTN, B.LqAttn), (B._RESIDUAL, B.LqResidual)):
        assert s.size == C.sizeof(c)
    assert get(B.lq_kvbatch(1, 2, 3, 4, 5, 6)) == [1, 2, 6, 3, 4, 5] and get(B.lq_kvbatch(1, 2, 3, 4, 5))[2] is None
    assert get(B.lq_kvrows(1, (2, 3, 4), None, (5, 6, -7))) == [1, None, 2, 3, 4, 5, 6, -7]
    assert get(B.lq_attn(1, (2, -3), 4, (5, 6), 7, 0.5, False, 8, 9)) == [1, 4, 2, -3, 5, 6, 7, 0, 8, 9, 0.5]
    assert get(B.lq_residual(1, 2, 3, 4, 5, 6, 7, 1, 8, 0.25, 9, 2, 10, 11, 12, 13, 14, 0.125, 1, 0, 1, 0, (21, 22, 23, 24), 5)) == \
        [3, 6, 4, 5, 21, 22, 23, 24, 8, 10, 11, 9, 12, 13, 14, 1, 2, 7, 1, 2, 1, 0, 1, 0, 0.25, 0.125, 5]
