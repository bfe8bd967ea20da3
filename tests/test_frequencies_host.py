"""Frequencies of position tables: the host code that forms them, compiled on its own, against 90 decimal digits.  No GPU needed."""
import ctypes as C
import os
import subprocess
from decimal import Decimal, getcontext

import pytest

from paper_2609_12378_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211707")
SOURCE = """
#include "frequencies.cuh"
extern "C" void frequencies(const ckks_rotary_scaling *f, double few, double many, double *hi, double *lo) { rotary_frequencies(*f, few, many, hi, lo); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("frequencies")
    (d / "f.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_12378_b200", "csrc"),
                    "-o", str(d / "f.so"), str(d / "f.cpp")], check=True)
    f = C.CDLL(str(d / "f.so")).frequencies
    f.restype = None
    f.argtypes = [C.POINTER(binding.CRotaryScaling), C.c_double, C.c_double, C.c_void_p, C.c_void_p]

    def run(rot, theta, kind, factor, length, few, many):
        s = binding.CRotaryScaling(binding.ROTARY_SCALINGS[kind], rot, theta, factor, length, few, many, 1.0)
        hi, lo = (C.c_double * (rot // 2))(), (C.c_double * (rot // 2))()
        f(C.byref(s), few, many, hi, lo)
        return list(hi), list(lo)
    return run


def angles(rot, theta, kind, factor, length, few, many):
    """Angle per position of every pair, from the definition; all arguments are the doubles that the library gets."""
    getcontext().prec = 90
    getcontext().Emin, getcontext().Emax = -10 ** 6, 10 ** 6
    D = Decimal
    t, f = D(theta), D(factor)
    if kind == "base":
        t = t * f ** (D(rot) / (rot - 2))
    w = [(-2 * j * t.ln() / rot).exp() for j in range(rot // 2)]
    if kind == "linear":
        return [x / f for x in w]
    if kind in ("bands", "ramp"):
        def blend(x, keep):
            keep = min(D(1), max(D(0), keep))
            return keep * x + (1 - keep) * x / f
        if kind == "bands":
            return [blend(x, (D(length) * x / (2 * PI) - D(few)) / (D(many) - D(few))) for x in w]
        at = [rot * (D(length) / (2 * PI * D(b))).ln() / (2 * t.ln()) for b in (many, few)]
        a, b = max(at[0].to_integral_value(rounding="ROUND_FLOOR"), D(0)), min(at[1].to_integral_value(rounding="ROUND_CEILING"), D(rot - 1))
        return [blend(x, 1 - (j - a) / max(b - a, D(0.001))) for j, x in enumerate(w)]
    return w


@pytest.mark.parametrize("rot", [2, 4, 6, 64, 96, 128, 250, 256])
@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1.0 + 2.0 ** -52, 1.5, 2.0, 4.0, 1e9, 1.7e308])
@pytest.mark.parametrize("kind,factor,length,few,many", [("none", 1.0, 0.0, 1.0, 4.0), ("linear", 4.0, 0.0, 1.0, 4.0), ("linear", 7.3, 0.0, 1.0, 4.0),
                                                         ("base", 8.0, 0.0, 1.0, 4.0), ("base", 1.0, 0.0, 1.0, 4.0), ("base", 1e300, 0.0, 1.0, 4.0),
                                                         ("bands", 8.0, 8192.0, 1.0, 4.0), ("bands", 3.7, 1e308, 0.3, 4.1), ("bands", 3.7, 1e-9, 0.3, 4.1),
                                                         ("ramp", 32.0, 8192.0, 1.0, 32.0), ("ramp", 5.1, 100.0, 1.0, 32.0)])
def test_frequencies_to_two_doubles(lib, rot, theta, kind, factor, length, few, many):
    """Relative to the angle: the powers carry 2^-115 or better, and each of at most ten operations on sums of two doubles rounds by at most
    2^-103: below 2^-99.  Next to the smallest double an operation's parts, four at most, are rounded to multiples of 2^-1074 besides: ten
    operations and the factor pi of this comparison make less than 40 * 4 * 2^-1075 < 2^-1067."""
    if kind == "base" and rot < 4:
        rot = 4
    hi, lo = lib(rot, theta, kind, factor, length, few, many)
    want = angles(rot, theta, kind, factor, length, few, many)
    for j, w in enumerate(want):
        got = (Decimal(hi[j]) + Decimal(lo[j])) * PI
        assert abs(got - w) <= w * Decimal(2) ** -99 + Decimal(2) ** -1067, (j, float(w), float((got - w) / w) if w else got)


def test_a_far_position_is_as_exact_as_a_near_one(lib):
    """Position 2^50 times a frequency's error stays below 2^-49, for every pair and not for the first alone."""
    for kind, factor in (("none", 1.0), ("linear", 3.0), ("base", 8.0), ("bands", 8.0), ("ramp", 32.0)):
        few, many = (1.0, 4.0) if kind == "bands" else (1.0, 32.0)
        a = (128, 500000.0, kind, factor, 8192.0, few, many)
        hi, lo = lib(*a)
        for j, w in enumerate(angles(*a)):
            assert abs((Decimal(hi[j]) + Decimal(lo[j])) * PI - w) * 2 ** 50 < Decimal(2) ** -49, (kind, j)


def test_bounds_next_to_the_smallest_double(lib):
    """Numbers there have few bits (the distance of the bounds 45, so that a part is off by 2^-44), and one over their distance is infinite."""
    hi, lo = lib(8, 10000.0, "bands", 4.0, 1.2e-309, 1e-310, 3e-310)
    want = angles(8, 10000.0, "bands", 4.0, 1.2e-309, 1e-310, 3e-310)
    for j, w in enumerate(want):
        assert abs((Decimal(hi[j]) + Decimal(lo[j])) * PI - w) <= w * Decimal(2) ** -40, j
