"""The polynomial of csrc/act.h for the normal distribution's tail, in 64 bits: f(z) = e^(z^2 / 2) erfc(|z| / sqrt 2) / 2 in t = 1 / (1 + A |z|)."""
import math
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_06079_amd", "csrc", "act.h")


def polynomial():
    """(A, coefficients, the highest power first) as the source has them."""
    body = open(SOURCE).read().split("Normal normal(float z)")[1].split("f *= e")[0]
    a = float(re.search(r"A = ([\d.]+)f", body).group(1))
    first = re.search(r"float f = (-?[\d.e-]+)f;", body).group(1)
    return a, [float(c) for c in [first] + re.findall(r"fmaf\(f, t, (-?[\d.e-]+)f\)", body)]


def test_fit():
    """Off by 2.1e-8 of f at most, with coefficients that fp32 holds."""
    a, c = polynomial()
    assert len(c) == 10 and all(float(np.float32(x)) == x for x in c)
    z = np.concatenate([np.linspace(0, 15.6, 20001), np.linspace(0, 1, 5001)])
    t = 1 / (1 + a * z)
    p = np.polyval(c, t)
    f = np.array([math.erfc(x / math.sqrt(2)) for x in z]) * np.exp(z * z / 2) / 2     # 64 bits: off by 1e-13
    assert np.max(np.abs(p / f - 1)) <= 2.1e-8


def test_what_rounding_counts():
    """The factors that the bounds of the GPU tests take: f changes by at most 2.33 times what t changes by, and the partial sums of the polynomial, each behind the powers of t that follow it,
    are together at most 4.1 f."""
    a, c = polynomial()
    z = np.linspace(0, 15, 20001)
    t = 1 / (1 + a * z)
    p, d, partial = np.full_like(t, c[0]), np.zeros_like(t), []
    for x in c[1:]:
        d, p = d * t + p, p * t + x
        partial.append(np.abs(p))
    assert np.max(np.abs(d * t / p)) <= 2.33
    assert np.max(sum(q * t ** (len(partial) - 1 - i) for i, q in enumerate(partial)) / np.abs(p)) <= 4.1
