"""GPU: activations of fp32 arguments with fp32 results, by the size of their relative errors (test_gpu_act.py bounds them against the argument alone).  U is half a step, 2^-24 relative.

SiLU.  p = 1 / (1 + e^-z): the power and the reciprocal are off by one step each (2 U), the power's factor is rounded twice near 1 (2 U), the sum once (U), and z p once more (U): 8 U.  What is left out
of the power's argument is known exactly, so no term grows with |z|.  The slope p + v (1 - p): 8 U of p and of 2 |v|.

GELU for z <= 0 is z f(|z|) e^(-z^2 / 2).  f (test_act_polynomial.py): the fit 2.1e-8 = 0.36 U, t's last rounding 2.33 U, the rounding of A |z| behind it U, partial sums 4.1 U; the power 2 U, its product with
f U, z's U; and the power's argument z^2 / 2 is rounded as a square, as a product and in its constant, 2.3 U of it together: (12 + 1.2 z^2) U.  For z > 0 it is z (1 - f e): that times f e / (1 - f e), and 2 U.

A product's activation (canz_linear) has neither correction.  SiLU: the power's argument is off by U of its size, and its constant by 0.22 U: (6 + 1.3 |z|) U.  GELU: t is off by a rounding of 1 + A |z| and a
step of the reciprocal, 3 U, which count 7 U: (16 + 1.2 z^2) U.

A power, p or Phi below 2^-126 may be flushed to 0, which takes (1 + |z|) 2^-125 at most."""
import math

import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, Mat, stream
from tests.test_gpu_linear import call

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def run(canz, kind, z):
    """(values, slopes) of the kernels."""
    import torch
    n = len(z)
    g, one, out, dg = Mat(1, n, F32, values=z[None]), Mat(1, n, F32, values=np.ones((1, n))), Mat(1, n, F32), Mat(1, n, F32)
    canz.canz_act_forward([canz.Act(rows=1, cols=n, gate=g, out=out, act=kind, dtype=F32)], stream())
    canz.canz_act_backward([canz.ActGrad(rows=1, cols=n, dout=one, gate=g, dgate=dg, act=kind, dtype=F32, in_dtype=F32)], stream())
    torch.cuda.synchronize()
    return out.get()[0], dg.get()[0]


def arguments(lo, hi):
    rng = np.random.default_rng(11)
    return np.concatenate([np.linspace(lo, hi, 20000), rng.uniform(lo, hi, 20000)]).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("lo,hi", [(-85, -14), (-14, -8), (-8, -2), (-2, 0), (0, 2), (2, 80)])
def test_silu(canz, lo, hi):
    z = arguments(lo, hi)
    got, slope = run(canz, L.SILU, z)
    p = 1 / (1 + np.exp(-z))
    flush = (1 + np.abs(z)) * 2.0 ** -125
    assert (np.abs(got - z * p) <= 8 * U * np.abs(z * p) + flush).all()
    assert (np.abs(slope - (p + z * p * (1 - p))) <= 8 * U * (p + 2 * np.abs(z * p)) + flush).all()


@pytest.mark.parametrize("lo,hi", [(-13, -8), (-8, -4), (-4, -2), (-2, -0.5), (-0.5, 0), (0, 0.5), (0.5, 2), (2, 30)])
def test_gelu(canz, lo, hi):
    z = arguments(lo, hi)
    got, slope = run(canz, L.GELU, z)
    tail, phi = 0.5 * _erfc(np.abs(z) / math.sqrt(2)), np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    p = np.where(z > 0, 1 - tail, tail)
    rel = (12 + 1.2 * z * z) * U
    err = np.where(z > 0, tail * rel + 2 * U, tail * rel)     # of Phi
    flush = (1 + np.abs(z)) * 2.0 ** -125
    assert (np.abs(got - z * p) <= np.abs(z) * err + flush).all()
    # the slope's second part: z times a constant, times the power (2 U, its argument as above), one sum
    assert (np.abs(slope - (p + z * phi)) <= err + np.abs(z) * phi * (5 + 1.2 * z * z) * U + U * np.abs(p + z * phi) + flush).all()


def test_gelu_near_zero_in_the_mean(canz):
    """-1/2 <= z < 0.  Roundings that do not depend on one another, each anywhere within its bound b, have the mean square b^2 / 3.  Here t lies in 0.85 .. 1, where half a step is U / 2: 1.26 U of f (0.73 U in the
    mean); the polynomial's last three partial sums are rounded by 0.62 U each, the ones before by 0.4 U together (0.66); the power by one step below 1, 1.06 U (0.61), its product with f by 0.62 (0.36),
    z's by 0.75 (0.42); the fit 0.36: in the mean 1.33 U.  Allowed: 1.5 U."""
    z = arguments(-0.5, 0)
    z = z[z < 0]
    got, _ = run(canz, L.GELU, z)
    want = z * 0.5 * _erfc(-z / math.sqrt(2))
    assert math.sqrt(np.mean((got / want - 1) ** 2)) <= 1.5 * U


def test_silu_far_below_zero_in_the_mean(canz):
    """Six roundings of 8 U together (power 2, factor 1 and 1, sum 1, reciprocal 2, product 1): sqrt(12 / 3) = 2 U in the mean at most."""
    z = arguments(-80, -8)
    got, _ = run(canz, L.SILU, z)
    want = z / (1 + np.exp(-z))
    assert math.sqrt(np.mean((got / want - 1) ** 2)) <= 2 * U


@pytest.mark.parametrize("kind,lo,hi", [(L.SILU, -80, 20), (L.GELU, -12, 12)])
def test_in_a_product(canz, kind, lo, hi):
    """z = a + bias is known here: k = 1, whole numbers a in bf16 and fractions in fp32, one rounding."""
    a, bias = np.arange(lo, hi, dtype=np.float64)[:, None], np.random.default_rng(12).uniform(0, 1, 999).astype(np.float32).astype(np.float64)
    m, n = len(a), len(bias)
    c = Mat(m, n, F32)
    call(canz, [canz.Linear(m=m, n=n, k=1, a=[Mat(m, 1, BF16, values=a)], b=[Mat(n, 1, BF16, values=np.ones((n, 1)))], c=[c], bias=[Mat(1, n, F32, values=bias[None])], out_dtype=F32, act=kind)])
    z = (a + bias).astype(np.float32).astype(np.float64)
    want = z / (1 + np.exp(-z)) if kind == L.SILU else z * 0.5 * _erfc(-z / math.sqrt(2))
    tail = 0.5 * _erfc(np.abs(z) / math.sqrt(2))
    rel = (16 + 1.2 * z * z) * U
    bound = np.abs(want) * (6 + 1.3 * np.abs(z)) * U if kind == L.SILU else np.abs(z) * np.where(z > 0, tail * rel + 2 * U, tail * rel)
    assert (np.abs(c.get() - want) <= bound + (1 + np.abs(z)) * 2.0 ** -125).all()


def test_infinite_and_large_arguments(canz):
    z = np.array([np.inf, -np.inf, np.nan, 3e38, -3e38, 1e19, -1e19, 16.5, -16.5, 127.0, -127.0, -0.0, 0.0, 2.0 ** -140, -2.0 ** -140], np.float32).astype(np.float64)
    import torch
    for kind in (L.SILU, L.GELU):
        n = len(z)
        g, one, out, dg = Mat(1, n, F32, values=z[None]), Mat(1, n, F32, values=np.ones((1, n))), Mat(1, n, F32), Mat(1, n, F32)
        canz.canz_act_forward([canz.Act(rows=1, cols=n, gate=g, out=out, act=kind, dtype=F32)], stream())
        canz.canz_act_backward([canz.ActGrad(rows=1, cols=n, dout=one, gate=g, dgate=dg, act=kind, dtype=F32, in_dtype=F32)], stream())
        torch.cuda.synchronize()
        v, d = out.view().cpu().numpy()[0], dg.view().cpu().numpy()[0]
        assert v[0] == np.inf and np.isnan(v[1]) and np.isnan(v[2]) and np.isnan(d[2])     # -inf times 0, as the formula has it
        assert (v[[3, 5, 9]] == z[[3, 5, 9]]).all() and abs(v[7] - 16.5) <= 2e-6 and (d[[3, 5, 9]] == 1).all()
        assert (v[[4, 6]] == 0).all() and (np.abs(v[[8, 10]]) <= 2e-6).all() and (d[[4, 6]] == 0).all()
        assert (v[[11, 12]] == 0).all() and np.signbit(v[11]) and (np.abs(d[11:15] - 0.5) <= 4 * U).all() and (np.abs(v[13:15] - z[13:15] / 2) <= 2.0 ** -149).all()
