"""Whether heads of a call lie on one place, on the CPU: against every pair of places of small layouts, and the layouts that programs have."""
import ctypes as C
import itertools
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "lq_heads_places.h"
extern "C" int collide(const LqRuns* a) { return lq_runs_collide(*a); }
extern "C" int meet(const LqRuns* a, const LqRuns* b) { return lq_runs_meet(*a, *b); }
"""
APART, SHARED, ENTANGLED = 0, 1, 2


class Runs(C.Structure):
    _fields_ = [("at", C.c_uint64), ("steps", C.c_int64 * 3), ("counts", C.c_int64 * 3), ("bytes", C.c_int64)]


def runs(at, steps, counts, nbytes):
    return Runs(at, (C.c_int64 * 3)(*(s if n > 1 else 0 for s, n in zip(steps, counts))), (C.c_int64 * 3)(*counts), nbytes)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("places")
    (d / "places.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_18117_b200", "csrc"),
                    str(d / "places.cpp"), "-o", str(d / "places.so")], check=True)
    so = C.CDLL(str(d / "places.so"))
    return lambda a: so.collide(C.byref(a)), lambda a, b: so.meet(C.byref(a), C.byref(b))


def places(r):
    """The first byte of each run."""
    return [r.at + sum(s * i for s, i in zip(r.steps, at)) for at in itertools.product(*(range(n) for n in r.counts))]


def test_small_layouts_against_every_pair(lib):
    collide, meet = lib
    rng = np.random.default_rng(1)
    seen = {(f, v): 0 for f in "cm" for v in (0, 1)}
    for _ in range(6000):
        def one(at):
            return runs(at, rng.integers(-12, 13, 3) * 16, rng.integers(1, 5, 3), int(rng.choice([1, 16, 32, 48])))
        a, b = one(10000), one(10000 + 16 * int(rng.integers(-30, 31)))
        if rng.random() < 0.4:                             # the same rows, other heads
            b = runs(b.at, [a.steps[0] or 16, a.steps[1] or 16, b.steps[2]], [a.counts[0], a.counts[1], b.counts[2]], b.bytes)
        pa, pb = np.sort(places(a)), np.array(places(b))
        want = int(pa.size > 1 and np.diff(pa).min() < a.bytes)
        assert collide(a) == want, (list(a.steps), list(a.counts), a.bytes)
        seen["c", want] += 1
        gap = pb[None] - pa[:, None]
        want = int(((gap > -b.bytes) & (gap < a.bytes)).any())
        assert meet(a, b) == want and meet(b, a) == want, (a.at, b.at, list(a.steps), list(b.steps), list(a.counts), list(b.counts), a.bytes, b.bytes)
        seen["m", want] += 1
    assert min(seen.values()) > 300, seen                  # both answers, often


def test_layouts_that_programs_have(lib):
    collide, meet = lib
    D, h, hk, S, Bn = 128 * 2, 32, 8, 32760, 16
    at = 1 << 40
    row = (h + 2 * hk) * D
    q, k = runs(at, (S * row, row, D), (Bn, S, h), D), runs(at + h * D, (S * row, row, D), (Bn, S, hk), D)         # inside the projection
    assert collide(q) == APART and collide(k) == APART and meet(q, k) == APART and meet(k, q) == APART
    assert meet(q, q) == SHARED and meet(q, runs(at + (h - 1) * D, (S * row, row, D), (Bn, S, hk), D)) == SHARED
    heads = runs(at, (2 * h * S * D, D, S * D), (Bn, S, h), D)                                                     # heads apart, K behind Q of each sequence
    other = runs(at + h * S * D, (2 * h * S * D, D, S * D), (Bn, S, h), D)
    assert collide(heads) == APART and meet(heads, other) == APART
    assert meet(heads, runs(other.at - 16, other.steps, other.counts, D)) == SHARED
    woven = runs(at + D, (S * h * 2 * D, h * 2 * D, 2 * D), (Bn, S, h), D)                                         # a query beside its key
    assert meet(runs(at, woven.steps, woven.counts, D), woven) == APART and meet(runs(at, woven.steps, woven.counts, D + 1), woven) == SHARED
    back = runs(at, (-S * row, -row, -D), (Bn, S, h), D)
    assert collide(back) == APART and meet(back, runs(at, (S * row, row, D), (Bn, S, h), D)) == SHARED


def test_outputs_of_two_dimensions_on_one_place(lib):
    collide, _ = lib
    assert collide(runs(0, (0, 128, 128), (1, 4, 2), 128)) == SHARED                       # the next row's first head is this row's second
    assert collide(runs(0, (0, 256, 128), (1, 4, 3), 128)) == SHARED
    assert collide(runs(0, (1024, 256, 128), (2, 5, 2), 128)) == SHARED                    # the next sequence begins in the last row
    assert collide(runs(0, (0, 512, 384), (1, 3, 2), 128)) == APART                        # woven, but every place once
    assert collide(runs(0, (0, 512, 384), (1, 4, 5), 128)) == SHARED                       # 3 x 512 = 4 x 384
    assert collide(runs(0, (0, 1 << 33, 16), (1, (1 << 31) - 1, 2), 16)) == SHARED         # no memory is as large


def test_what_cannot_be_told_in_few_steps_is_said_to_be_so(lib):
    """Each side's rows hit the other's steps at a different place each time, all of them just beside its heads: apart, but found so only by looking
    at half a million places."""
    _, meet = lib
    a = runs(0, (0, 1 << 20, 0), (1, 1 << 20, 1), 16)
    b = runs(1 << 19, (0, (1 << 20) + 32, 0), (1, 1 << 14, 1), 16)             # 2^19 + 32 i over i < 2^14: behind a head's end, before the next one's
    assert meet(a, b) == APART
    c = runs(1 << 19, (0, (1 << 20) + 1, 0), (1, (1 << 19) - 16, 1), 16)
    assert meet(a, c) == ENTANGLED


def test_the_longest_rows_take_few_steps(lib):
    collide, meet = lib
    n = (1 << 31) - 1
    a = runs(1 << 20, (0, 16, 0), (1, n, 1), 16)
    assert collide(a) == APART and meet(a, runs((1 << 20) + 16 * n, (0, 16, 0), (1, n, 1), 16)) == APART
    assert meet(a, runs((1 << 20) + 16 * (n - 1), (0, 0, 0), (1, 1, 1), 16)) == SHARED
    # two combs whose teeth fall beside one another, in step and out of step
    comb = runs(1 << 20, (0, 64, 0), (1, n // 4, 1), 16)
    assert meet(comb, runs((1 << 20) + 32, (0, 64, 0), (1, n // 4, 1), 16)) == APART
    assert meet(comb, runs((1 << 20) + 32, (0, 128, 0), (1, n // 8, 1), 16)) == APART
    assert meet(comb, runs((1 << 20) + 32, (0, 192, 64), (1, n // 16, 3), 16)) == APART
    assert meet(comb, runs((1 << 20) + 48, (0, 192, 64), (1, n // 16, 3), 17)) == SHARED
    assert meet(comb, runs((1 << 20) + 32, (0, 80, 0), (1, n // 8, 1), 16)) == SHARED
