"""The angle of a pair at a position: the part of a turn against whole numbers.

A frequency's turn a position is held in whole 2^-64 of a turn, the sum of two roundings (half a step each; what f / 2 pi is off by itself, 2^-104 of at most 2^38
turns, is 2^-66): off by 1 + 2^-2 steps at most, |pos| times that at a position, and a step more where a half turn saturates.  The fp32 number of half turns
is rounded once, 2^-24 of itself.
"""
import ctypes
import os
import random
import subprocess
from fractions import Fraction

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BITS = 400


def _inverse_of_two_pi():
    """floor(2^BITS / 2 pi), pi by Machin's formula."""
    def arctan_of_inverse(x, one):
        total = term = one // x
        n, sign = 3, -1
        while term:
            term //= x * x
            total += sign * (term // n)
            n, sign = n + 2, -sign
        return total
    one = 1 << (BITS + 100)
    pi = 4 * (4 * arctan_of_inverse(5, one) - arctan_of_inverse(239, one))
    return (one << BITS) // (2 * pi)


INV_TWO_PI = _inverse_of_two_pi()


def part_of_turn(pos: int, f: float) -> Fraction:
    """between -1/2 and 1/2, to 2^-300"""
    t = Fraction(f) * pos * Fraction(INV_TWO_PI, 1 << BITS)
    return t - round(t)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("native") / "angle.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2408_11746_b200", "csrc"),
                    os.path.join(ROOT, "tests", "native", "angle.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.turn_a_position.restype, lib.turn_a_position.argtypes = ctypes.c_uint64, [ctypes.c_float]
    lib.half_turns.restype, lib.half_turns.argtypes = ctypes.c_float, [ctypes.c_float, ctypes.c_int]
    return lib


@pytest.mark.parametrize("top", [1e-9, 1.0, 1000.0, 2.0 ** 20, 2.0 ** 40])
def test_parts_of_a_turn(lib, top):
    rng = random.Random(int(top))
    for i in range(4000):
        pos = rng.choice([rng.randint(-(1 << 31), (1 << 31) - 1), (1 << 31) - 1 - rng.randint(0, 9), -(1 << 31), rng.randint(0, 40000), 0, 1])
        f = float(np.float32(rng.choice([top, top * rng.random(), -top * rng.random(), top * 10000.0 ** -rng.random(), 0.0])))
        got = Fraction(lib.half_turns(f, pos)) / 2
        off = got - part_of_turn(pos, f)
        off -= round(off)              # half a turn is minus half a turn
        assert abs(off) <= Fraction(2.25 * abs(pos) * 2.0 ** -64) + abs(got) * Fraction(2.0 ** -24), (pos, f)
        assert abs(got) <= Fraction(1, 2)
        step = Fraction(lib.turn_a_position(f), 1 << 64) - part_of_turn(1, f)
        assert abs(step - round(step)) <= Fraction(2.25 * 2.0 ** -64)


def test_frequencies_at_the_ends(lib):
    assert lib.half_turns(0.0, (1 << 31) - 1) == 0.0 and lib.half_turns(1.0, 0) == 0.0 and abs(lib.half_turns(1e-45, 7)) < 1e-18
    for f in (3.4e38, -3.4e38, float("inf"), float("nan")):        # no angle is claimed; nothing is undefined
        assert abs(lib.half_turns(f, (1 << 31) - 1)) <= 1.0
