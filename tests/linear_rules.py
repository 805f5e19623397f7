"""The rules by which canz_linear takes its kernels, asked from csrc/linear_rules.h itself: a test of one of them then says that its shapes still reach it."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_06079_amd", "csrc")
SOURCE = """#include "linear_rules.h"
extern "C" {
int few(long long m, int a_trans, int b_trans) { return canz::linear_few(m, a_trans, b_trans); }
int parts(long long m, long long n, long long k) { return canz::linear_parts(m, n, k); }
int large_tiles(long long large, long long small, long long steps) { return canz::linear_large_tiles(large, small, steps); }
}
"""


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
    r.few.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    r.parts.argtypes = r.large_tiles.argtypes = [ctypes.c_longlong] * 3
    return r


def few(m, a_trans=False, b_trans=False):
    return bool(lib().few(m, a_trans, b_trans))


def parts(m, n, k):
    return lib().parts(m, n, k)


def large_tiles(m, n, k):
    """Whether a product that is alone in its call (and not one of few rows) takes tiles of 256 x 256."""
    p = parts(m, n, k)
    large, small = p * (-(-m // 256) * -(-n // 256)), p * (-(-m // 128) * -(-n // 128))
    steps = -(-k // 32)
    return bool(lib().large_tiles(large, small, -(-(steps * (small // p)) // small)))
