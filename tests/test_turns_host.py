"""Frequencies as 64-bit fractions of a turn, on the CPU, against whole numbers of 400 bits."""
import ctypes as C
import os
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = '#include "lq_turns.h"\nextern "C" uint64_t turn(double f) { return lq_turn_fraction(f); }\n'


def pi(bits=420):
    """pi from Machin's formula, within 2^-400."""
    def arctan_of_inverse(x):
        term, total, n = (1 << bits) // x, 0, 1
        while term:
            total += (term // n) * (1 if n % 4 == 1 else -1)
            term, n = term // (x * x), n + 2
        return total
    return Fraction(4 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)), 1 << bits)


@pytest.fixture(scope="module")
def turn(tmp_path_factory):
    d = tmp_path_factory.mktemp("turns")
    (d / "turns.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_18117_b200", "csrc"),
                    str(d / "turns.cpp"), "-o", str(d / "turns.so")], check=True)
    f = C.CDLL(str(d / "turns.so")).turn
    f.argtypes, f.restype = [C.c_double], C.c_uint64
    return f


def test_fractions_of_a_turn(turn):
    rng = np.random.default_rng(0)
    two_pi = 2 * pi()
    values = [0.0, -0.0, 1.0, -1.0, 2 * np.pi, 100.0, 1e6, -1e6, 1e15 + 0.125, 2.0 ** 63, np.nextafter(2.0 ** 64, 0), 5e-324, 1e-300, 2.0 ** -60,
              2.0 ** -61, 2.0 ** -62, 2.0 ** -63, 2.0 ** -64]
    values += list(rng.standard_normal(2000) * 2.0 ** rng.integers(-70, 62, 2000))
    for v in values:
        exact = Fraction(float(v)) / two_pi * 2 ** 64
        off = (turn(v) - exact) % 2 ** 64                  # 2^64 is no turn at all
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 60), v
        assert (turn(-v) + turn(v)) % 2 ** 64 == 0


def test_frequencies_without_an_angle_are_refused():
    for v, code in ((2.0 ** 64, 2), (-1e30, 2), (1.7e308, 2), (np.inf, 6), (-np.inf, 6), (np.nan, 6)):
        with pytest.raises(B.LqError) as e:
            B.lq_rope_create(B.lq_rope_config_default([8]), 0, np.array([1.0, v, 0.5, 0.0]))
        assert e.value.code == code, v
    with pytest.raises(B.LqError) as e:                    # theta^(-3 / 4) of the last pair: 3e22
        B.lq_rope_create(B.lq_rope_config_default([8], theta=1e-30), 0)
    assert e.value.code == 2
