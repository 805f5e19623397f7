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
long long whole_rounds(long long large, long long steps) { return canz::linear_whole_rounds(large, steps); }
int few_width(long long n, int pre) { return canz::linear_few_width(n, pre); }
int alone(long long longest, long long all_steps) { return canz::linear_alone(longest, all_steps); }
int cus() { return canz::LINEAR_CU; }
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
    r.few_width.argtypes, r.alone.argtypes = [ctypes.c_longlong, ctypes.c_int], [ctypes.c_longlong] * 2
    r.whole_rounds.argtypes, r.whole_rounds.restype = [ctypes.c_longlong] * 2, ctypes.c_longlong
    return r


def few(m, a_trans=False, b_trans=False):
    return bool(lib().few(m, a_trans, b_trans))


def parts(m, n, k):
    return lib().parts(m, n, k)


def _tiles(m, n, k):
    p = parts(m, n, k)
    large, small = p * (-(-m // 256) * -(-n // 256)), p * (-(-m // 128) * -(-n // 128))
    return large, small, -(-(-(-k // 32) * (small // p)) // small)


def large_tiles(m, n, k):
    """Whether a product that is alone in its call (and not one of few rows) takes tiles of 256 x 256."""
    return bool(lib().large_tiles(*_tiles(m, n, k)))


def quarters(m, n, k):
    """How many of its 256 x 256 tiles are done in quarters by small ones behind the last whole round."""
    large, _, steps = _tiles(m, n, k)
    rounds = lib().whole_rounds(large, steps) if large_tiles(m, n, k) else 0
    return large - rounds * lib().cus() if rounds else 0


def one_small_tile_to_a_cu(m, n, k):
    return not large_tiles(m, n, k) and -(-_tiles(m, n, k)[1] // 8) * 8 <= lib().cus()


def few_width(n, pre):
    """Which blocks (16, 32 or 64 rows of B) a product of few rows takes, with an image of z or without."""
    return 16 << lib().few_width(n, pre)


def one_launch(shapes):
    """(whether a launch of these products, not of few rows and of one orientation, takes tiles of 256 x 256; small tiles; whether a ring of four stages does them, one to a CU)."""
    tiles = []
    for m, n, k in shapes:
        p, steps = parts(m, n, k), -(-k // 32)
        ends = [z * steps // p // 4 * 4 for z in range(p)] + [steps]
        tiles += [(-(-m // 256) * -(-n // 256), -(-m // 128) * -(-n // 128), b - a) for a, b in zip(ends, ends[1:])]
    large, small, all_steps = sum(t[0] for t in tiles), sum(t[1] for t in tiles), sum(t[1] * t[2] for t in tiles)
    share = sum(-(-t[1] // 8) for t in tiles) * 8
    four = share <= lib().cus() or bool(lib().alone(max(t[2] for t in tiles), all_steps))
    return bool(lib().large_tiles(large, small, -(-all_steps // small))), small, four
