"""Sines and cosines of the rotation (csrc/rotate.hpp) against 64 bits, compiled for the CPU: the same operations on 32-bit floats, each rounded once."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06833_amd", "csrc")
PREFIX = "#define __device__\n#define __forceinline__ inline\n"
CALLS = r"""
extern "C" void quarters(const float *r, float *s, float *c, long n) { for (long i = 0; i < n; ++i) sincos_quarter(r[i], s[i], c[i]); }
extern "C" void angles(const int *p, double f, float *s, float *c, long n) { for (long i = 0; i < n; ++i) sincos_of((double)p[i], f, s[i], c[i]); }
"""
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("sines")
    text = open(os.path.join(CSRC, "rotate.hpp")).read()
    bodies = re.findall(r"^__device__ __forceinline__ void sincos_\w+\(.*?^}\n", text, re.M | re.S)
    assert len(bodies) == 2
    (d / "s.cpp").write_text(PREFIX + "".join(bodies) + CALLS)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-o", str(d / "s.so"), str(d / "s.cpp")], check=True)
    L = C.CDLL(str(d / "s.so"))
    L.quarters.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_long]
    L.angles.argtypes = [C.c_void_p, C.c_double, C.c_void_p, C.c_void_p, C.c_long]
    return L


def outputs(call, n, *args):
    s, c = np.empty(n, np.float32), np.empty(n, np.float32)
    call(*args, s.ctypes.data, c.ctypes.data, n)
    return s.astype(np.float64), c.astype(np.float64)


def test_a_quarter_turn(lib):
    """x = r pi / 2 is off by 2^-24 of itself for the constant and its product each, which turns to at most 2^-24 (pi / 4) (cos, sin) of the results; the last
    sums round by 2^-25 (results below 1; the cosine's up to 1 by 2^-25 too), the terms before them by less than 2^-25: below 2 * 2^-24 together."""
    rng = np.random.default_rng(0)
    r = np.concatenate([rng.uniform(-0.5, 0.5, 4_000_000), np.exp2(rng.uniform(-20, -1, 2_000_000)) * rng.choice([-1, 1], 2_000_000), [0.0, 0.5, -0.5]]).astype(np.float32)
    s, c = outputs(lib.quarters, r.size, r.ctypes.data)
    x = r.astype(np.float64) * (np.pi / 2)
    worst = max(np.abs(s - np.sin(x)).max(), np.abs(c - np.cos(x)).max()) / U
    print("largest errors, in 2^-24: sine %.3f, cosine %.3f" % (np.abs(s - np.sin(x)).max() / U, np.abs(c - np.cos(x)).max() / U))
    assert worst < 2.0
    # relative to the sine itself, which the rows near an angle of 0 have: the two roundings of x, the product's and the sum's
    some = r != 0
    assert (np.abs(s - np.sin(x))[some] / np.abs(np.sin(x))[some]).max() < 4 * U


def test_whole_turns(lib):
    """Far angles lose nothing but what r itself rounds, 2^-26 of a quarter turn (0.4 * 2^-24 radians): with a given r's 1.44 * 2^-24 still below 2 * 2^-24."""
    rng = np.random.default_rng(1)
    p = np.concatenate([rng.integers(-2 ** 31, 2 ** 31, 300_000), np.arange(-5, 6)]).astype(np.int32)
    for f in (1.0, 0.25, 1e-3, 1e-6, np.pi / 2 * (1 - 2.0 ** -30)):
        s, c = outputs(lambda a, b, d, n: lib.angles(a, f, b, d, n), p.size, p.ctypes.data)
        t = p.astype(np.longdouble) * np.longdouble(f)
        # the product in 64 bits is off by 2^-53 of itself, as is its share of a turn
        far = np.abs(p.astype(np.float64)) * f * 2.0 ** -52
        assert (np.abs(s - np.sin(t).astype(np.float64)) <= 2 * U + far).all()
        assert (np.abs(c - np.cos(t).astype(np.float64)) <= 2 * U + far).all()
