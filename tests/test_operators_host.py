"""Refusals of the adapters' and heads' entry points that need no GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B


def _code(f, *a):
    with pytest.raises(B.LqError) as e:
        f(*a)
    return e.value.code


def test_sizes_of_an_adapter_set():
    for bad in ((0, 8, 8, 1), (8, -8, 8, 1), (8, 8, 0, 1), (8, 8, 8, 0)):
        assert _code(B.lq_adapters_create, *bad) == 1, bad
    for bad in ((8200, 8, 8, 1), (12, 8, 8, 1), (8, 12, 8, 1), (8, 8, 129, 1), (8, 8, 8, 1024)):
        assert _code(B.lq_adapters_create, *bad) == 2, bad


def test_sizes_of_a_row_map():
    assert _code(B.lq_rowmap_create, 0, 1) == 1 and _code(B.lq_rowmap_create, 1, 0) == 1
    assert _code(B.lq_rowmap_create, 1, 1024) == 2 and _code(B.lq_rowmap_create, (1 << 24) + 1, 1) == 2


def test_null_handles():
    L = B.lib()
    assert L.lq_adapters_free(None) == 1 and L.lq_rowmap_free(None) == 1 and L.lq_rope_free(None) == 1
    assert L.lq_adapters_set(None, 0, 1, None, None, 1.0, None) == 1 and L.lq_rowmap_set(None, None, 1, None) == 1
    assert L.lq_adapters_forward(None, None, None, None, None, 0, None) == 1
    assert L.lq_qk_norm_rope(None, None, 64, 1, 1, 1, 1e-6, None, None, 0, 0, None) == 1
    assert L.lq_qkv_forward(None, None, None, 1, None, None, None, None, 0, None) == 1
    assert L.lq_rope_config_default(None, 0, None) == 1 and L.lq_rope_create(None, None, None, 0, None) == 1


def test_rotation_tables():
    cfg = lambda dims, **k: B.lq_rope_config_default(dims, **k)
    assert list(cfg([36, 36]).dims) == [36, 36, 0, 0] and cfg([36, 36]).axes == 2 and cfg([]).axes == 0
    assert _code(cfg, [8] * 5) == 1
    for bad in (cfg([7]), cfg([-2]), cfg([8], theta=0.0), cfg([8], theta=float("inf"))):
        assert _code(B.lq_rope_create, bad) == 1
    for bad in (cfg([258]), cfg([128, 130]), cfg([12], halves=True)):
        assert _code(B.lq_rope_create, bad) == 2
    assert _code(B.lq_rope_create, cfg([8, 8]), 0, None, np.array([0, 1, 2, 0, 0, 0, 0, 0])) == 1
    assert _code(B.lq_rope_create, cfg([8]), 0, np.array([0, 1, np.nan, 2.0])) == 6
    bad = cfg([8])
    bad.halves = 2
    assert _code(B.lq_rope_create, bad) == 1
    bad = cfg([8])
    bad.axes = 5
    assert B.lib().lq_rope_create(C.byref(bad), None, None, 0, C.byref(C.c_void_p())) == 1


def test_layouts_of_the_structures():
    """The binding's structures have the header's sizes (four bytes before theta, and at the end of the heads)."""
    assert C.sizeof(B.LqHeads) == 2 * 8 + 6 * 8 + 2 * 8 + 8 and C.sizeof(B.LqRopeConfig) == 7 * 4 + 4 + 8
    assert C.sizeof(B.LqQkv) == 6 * 4 + 6 * 8
