"""The rules by which canz_mx_product takes its kernels, asked from csrc/mx_rules.h itself: a test of one of them then says that its shapes still reach it."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_06079_amd", "csrc")
SOURCE = """#include "mx_rules.h"
extern "C" {
int large_tiles(long long large, long long small, long long ks) { return canz::mx_large_tiles(large, small, ks); }
int width(long long n) { return canz::width_of(n); }
int rounds_on_the_way(long long m, long long n, long long k) { return canz::mx_rounds_on_the_way(m, n, k); }
int parts(long long m, long long n, long long k) { return canz::mx_parts(m, n, k); }
int few_rows() { return canz::FEW_ROWS; }
}
"""
NARROW, MIDDLE, WIDE = 0, 1, 2


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
    for f in (r.large_tiles, r.width, r.rounds_on_the_way, r.parts):
        f.argtypes = [ctypes.c_longlong] * (1 if f is r.width else 3)
    return r


def width(n):
    return lib().width(n)


def rounds_on_the_way(m, n, k):
    return bool(lib().rounds_on_the_way(m, n, k))


def parts(m, n, k):
    return lib().parts(m, n, k)


def large_tiles(shapes):
    """Whether products of these (m, n, k), more than 64 rows each and at most 32 problems in all, take tiles of 256 x 256 in one call."""
    large = small = units = 0
    problems = 0
    for m, n, k in shapes:
        assert m > lib().few_rows()
        p, u = parts(m, n, k), -(-k // 128)
        t = -(-m // 128) * -(-n // 128)
        large += p * (-(-m // 256) * -(-n // 256))
        small += p * t
        units += t * u                       # the parts' units add up to the whole's
        problems += p
    assert problems <= 32
    return bool(lib().large_tiles(large, small, -(-units // small)))
