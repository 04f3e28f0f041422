"""The frequencies that rotary positions keep, against 50 decimal digits, within what the header promises of their angles."""
import ctypes
import decimal
import os
import subprocess
from decimal import Decimal

import pytest

from paper_2609_05228_gb300 import ace

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_05228_gb300", "csrc")
TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def turns(tmp_path_factory):
    """F_i of a description and a divisor, as ace_rope_create makes it."""
    d = tmp_path_factory.mktemp("angles")
    (d / "angles.cpp").write_text('#include "ace_angles.h"\nextern "C" uint64_t turn(const ace_rope_desc* D, int i, double divisor) {\n'
                                  "    return ace::rope_turn(ace::rope_frequency(*D, i) / divisor);\n}\n")
    lib = d / "angles.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(d / "angles.cpp"), "-o", str(lib)],
                   check=True)
    f = ctypes.CDLL(str(lib)).turn
    f.restype, f.argtypes = ctypes.c_uint64, [ctypes.POINTER(ace.ace_rope_desc), ctypes.c_int, ctypes.c_double]
    return f


def _exact(i, rot, base, scaling, factor, length, low, high):
    """f_i in turns and how many times the relative part of the bound counts."""
    base, factor, length, low, high = (Decimal(x) for x in (base, factor, length, low, high))
    t = (-2 * Decimal(i) / rot * base.ln()).exp()
    if scaling == "none":
        return t / TWO_PI, 1
    if scaling == "linear":
        return t / factor / TWO_PI, 1
    times = 1
    if scaling == "by_turns":
        g = (length * t / TWO_PI - low) / (high - low)
        times = factor * high / (high - low) if 0 < g < 1 else 1
    else:
        def index(turns):
            return rot * (length / (TWO_PI * turns)).ln() / (2 * base.ln())
        a = max(index(high).to_integral_value(decimal.ROUND_FLOOR), 0)
        z = min(index(low).to_integral_value(decimal.ROUND_CEILING), rot - 1)
        g = 1 - (i - a) / ((z if z != a else a + Decimal("0.001")) - a)
    g = min(max(g, 0), 1)
    return t * (g + (1 - g) / factor) / TWO_PI, times


KINDS = [("none", 1.0, 0.0, 1.0, 32.0), ("linear", 3.0, 0.0, 1.0, 32.0), ("by_turns", 8.0, 8192.0, 1.0, 4.0), ("by_turns", 40.0, 4096.0, 1.0, 32.0),
         ("by_index", 16.0, 4096.0, 1.0, 32.0)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("base", [100.0, 1e4, 5e5, 1e8, 1e30])
@pytest.mark.parametrize("rot", [2, 48, 80, 128, 256])
def test_kept_frequencies_are_within_the_stated_bound(turns, rot, base, kind):
    """A position's share of the bound, in 2^-64ths of a turn: one half, and (4 + ln base) 2^-53 f_i (one rounding of it for the divisor)."""
    scaling, factor, length, low, high = KINDS[kind]
    desc = ace.ace_rope_desc(256, rot, 0, 0, ace.ROPE_SCALINGS.index(scaling), base, factor, length, low, high, 1.0)
    with decimal.localcontext(decimal.Context(prec=60)):
        for i in range(rot // 2):
            for divisor in (1.0, 1.7):
                f, times = _exact(i, rot, base, scaling, factor, length, low, high)
                f /= Decimal(divisor)
                kept = Decimal(turns(ctypes.byref(desc), i, divisor))
                off = abs(kept - f * 2 ** 64)           # (f_i is below a turn)
                assert off <= Decimal("0.5") + (4 + Decimal(base).ln()) * times * f * 2 ** 11, (i, off)
