"""CPU test of when a row's probabilities are good enough against a fixed reference: the header that the kernels use, compiled for the host, and fp16's
roundings emulated around it."""
import ctypes as C
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16928_amd", "csrc")
SOURCE = """
#include "chunk_reach.h"
using namespace rtp;
extern "C" int in_reach(int f16, int held, float sum, int seen) { return chunk_in_reach(f16 != 0, held != 0, sum, seen); }
extern "C" int seen_among(int from, int end, int local, int sink, int lo, int hi) { return chunk_seen_among(from, end, local != 0, sink, lo, hi); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "a host C++ compiler is needed"
    d = tmp_path_factory.mktemp("reach")
    (d / "reach.cpp").write_text(SOURCE)
    so = str(d / "reach.so")
    subprocess.run([cxx, "-std=c++17", "-O2", "-shared", "-fPIC", "-w", "-D__host__=", "-D__device__=", "-D__forceinline__=inline", "-I", CSRC,
                    str(d / "reach.cpp"), "-o", so], check=True)
    L = C.CDLL(so)
    L.in_reach.argtypes = [C.c_int, C.c_int, C.c_float, C.c_int]
    return L


def test_keys_are_counted(lib):
    rng = random.Random(1)
    for _ in range(4000):
        start, n, sink, window, m = rng.randint(0, 40), rng.randint(0, 60), rng.choice([0, 0, 3, 20, 200]), rng.choice([0, 1, 9, 70]), rng.randint(-5, 110)
        hi, lo = min(m, rng.choice([m, 50])), m - window
        keys = range(start, start + n)
        assert lib.seen_among(start, start + n, 0, sink, lo, hi) == sum(k <= hi for k in keys)
        assert lib.seen_among(start, start + n, 1, sink, lo, hi) == sum(k <= hi and (k < sink or k > lo) for k in keys)


@pytest.mark.parametrize("spread", [0.0, 0.05, 0.5, 2.0])
def test_what_is_accepted_is_exact_enough(lib, spread):
    """Probabilities rounded to fp16 against a reference that the row does not see, values of +1 and -1 by the direction of every rounding, which nothing
    averages: what is accepted is within 2^-12 of the sum, beside the half step of probabilities above 2^-14."""
    rng, accepted, refused = np.random.default_rng(5), 0, 0
    for n in (1, 3, 40, 700, 8192, 100000):
        for below in np.arange(-4.0, 40.0, 0.25):                 # binades between the reference and the middle of what the row sees
            p = np.exp2(-below + spread * rng.standard_normal(n))
            with np.errstate(over="ignore"):
                P = p.astype(np.float16).astype(np.float64)
            total = P.sum()
            if not lib.in_reach(1, 0, float(total), n) or not np.isfinite(total):
                refused += 1
                continue
            accepted += 1
            v = np.where(P > p, 1.0, -1.0)
            exact = (p * v).sum() / p.sum()
            allowed = 2.0 ** -12 + 2.0 ** -11 * (p * np.abs(v - exact)).sum() / p.sum()
            assert abs((P * v).sum() / total - exact) <= 2 * allowed, (n, below)      # (|v - exact| is up to 2)
    assert accepted > 100 and refused > 100


def test_rows_that_see_their_reference_are_not_refused(lib):
    for n in (1, 1000, 1 << 20, 1 << 30):
        assert lib.in_reach(1, 1, 0.99, n) and lib.in_reach(0, 1, 0.99, n) and lib.in_reach(0, 0, 0.99, n)
    assert not lib.in_reach(1, 0, 2.0 ** -5, 8192)                # 8192 probabilities of 2^-18: 64 steps each
    assert not lib.in_reach(1, 0, 0.99, 100000)
    assert lib.in_reach(1, 0, 2.0 ** -5, 200) and lib.in_reach(0, 0, 2.0 ** -50, 8192)
    for held in (0, 1):
        for f16 in (0, 1):
            assert lib.in_reach(f16, held, 0.0, 0)                # a row that sees nothing there
            assert not lib.in_reach(f16, held, 0.0, 1) and not lib.in_reach(f16, held, float("nan"), 3)
