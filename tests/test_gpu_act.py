"""GPU: canz_act_forward and canz_act_backward against the fp64 oracle.

Bounds.  e^x is off by the rounding of its argument, 2 |x| 2^-24, and one step; 1 / v by one step.  So SiLU's p = 1 / (1 + e^-z) is off by at most (|z| + 4) 2^-22 of itself (a factor of two
in hand), its value z p likewise, and its slope p + v (1 - p) by (|p| + 2 |v|) times that.  GELU's Phi is off by the rounding of the argument, which counts z^2 2^-22 at most, and 16
steps of erfc: (z^2 + 16) 2^-22; its slope by that times |Phi| + |z phi|.  A p or Phi below 2^-126 may be flushed to 0,
which takes |z| 2^-126 from a value and (1 + |z|) 2^-126 from a slope (the first run showed it at z = -88.7: 88.7 2^-126 where 2^-124 was allowed for).  Products add 2^-23 each, and a result is
rounded once to its type.  NONE and RELU are exact but for the products."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, MX8, Image, Mat, close, held, image_of, same_image, stream

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 32), (7, 127), (5, 1000), (66, 1531), (2, 4096)]
FLUSH = 2.0 ** -124


def bounds(kind, z):
    """(fp32 error bound of act(z), of its slope)"""
    if kind == L.SILU:
        p = 1 / (1 + np.exp(-z))
        rel = (np.abs(z) + 4) * 2.0 ** -22
        return np.abs(z * p) * rel + (1 + np.abs(z)) * FLUSH, (p + 2 * np.abs(z * p)) * rel + (1 + np.abs(z)) * FLUSH
    if kind == L.GELU:
        rel = (z * z + 16) * 2.0 ** -22
        phi = np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        p = L.act(L.GELU, z) / np.where(z == 0, 1, z)
        p = np.where(z == 0, 0.5, p)
        return np.abs(z * p) * rel + (1 + np.abs(z)) * FLUSH, (p + np.abs(z) * phi) * rel + (1 + np.abs(z)) * FLUSH
    return np.zeros_like(z), np.zeros_like(z)


def inputs(rng, rows, cols, dtype):
    z = rng.standard_normal((rows, cols)) * 3
    z[rng.random((rows, cols)) < 0.05] *= 10
    z[rng.random((rows, cols)) < 0.02] = 0
    return held(z, dtype), held(rng.standard_normal((rows, cols)) * 2, dtype), held(rng.standard_normal((rows, cols)) * 1e-3, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", [L.NONE, L.SILU, L.GELU, L.RELU])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(canz, rows, cols, kind, dtype):
    import torch
    rng = np.random.default_rng(rows * 31 + cols + kind)
    gate, up, _ = inputs(rng, rows, cols, dtype)
    for with_up in (False, True):
        g, out, g8 = Mat(rows, cols, dtype, 3, 1, gate), Mat(rows, cols, dtype, 5, 3), Image(rows, cols)
        u, u8 = (Mat(rows, cols, dtype, 3, 2, up), Image(rows, cols)) if with_up else (None, None)
        canz.canz_act_forward([canz.Act(rows=rows, cols=cols, gate=g, up=u, out=out, gate8=g8, up8=u8, act=kind, dtype=dtype, ld_in=g.ld, ld_out=out.ld)], stream())
        torch.cuda.synchronize()
        want = L.gated(kind, gate, up if with_up else None)
        b, _ = bounds(kind, gate)
        close(out.get(), want, (b * np.abs(up) + np.abs(want) * 2 ** -23) if with_up else b, dtype)
        same_image(g8, gate)
        if with_up:
            same_image(u8, up)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("in_dtype", [F32, BF16, MX8])
@pytest.mark.parametrize("kind", [L.NONE, L.SILU, L.GELU, L.RELU])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(canz, rows, cols, kind, in_dtype, dtype):
    import torch
    rng = np.random.default_rng(rows * 37 + cols + kind)
    gate, up, dout = inputs(rng, rows, cols, min(in_dtype, BF16))
    dout = held(dout, dtype)
    if in_dtype == MX8:
        gate, up = L.eight(gate), L.eight(up)
    for with_up in (False, True):
        make = image_of if in_dtype == MX8 else lambda x: Mat(rows, cols, in_dtype, 3, 1, x)
        g, u = make(gate), make(up) if with_up else None
        d, dg, out = Mat(rows, cols, dtype, 5, 1, dout), Mat(rows, cols, dtype, 3, 3), Mat(rows, cols, dtype, 5, 2)
        du = Mat(rows, cols, dtype, 3, 1) if with_up else None
        canz.canz_act_backward([canz.ActGrad(rows=rows, cols=cols, dout=d, gate=g, up=u, dgate=dg, dup=du, out=out, act=kind, dtype=dtype, in_dtype=in_dtype,
                                             ld_in=dg.ld, ld_out=out.ld)], stream())
        torch.cuda.synchronize()
        b, bs = bounds(kind, gate)
        ru = up if with_up else np.ones_like(up)
        want_dg, want_du = L.gated_grad(kind, dout, gate, up if with_up else None)
        want = L.gated(kind, gate, up if with_up else None)
        close(dg.get(), want_dg, np.abs(dout * ru) * bs + np.abs(want_dg) * 2 ** -22 + FLUSH, dtype, "dgate")
        close(out.get(), want, b * np.abs(ru) + np.abs(want) * 2 ** -23, dtype, "out")
        if with_up:
            close(du.get(), want_du, np.abs(dout) * b + np.abs(want_du) * 2 ** -23 + FLUSH, dtype, "dup")


@pytest.mark.parametrize("kind", [L.SILU, L.GELU])
def test_gradient_against_differences(canz, kind):
    """(f(z + h) - f(z - h)) / 2h of the kernel's own forward pass with h = 2^-6: off by h^2 / 6 times the third derivative (at most 1) and by the values' errors over h."""
    import torch
    rng = np.random.default_rng(8)
    rows, cols, h = 20, 300, 2.0 ** -6
    z = held(rng.uniform(-6, 6, (rows, cols)), BF16)     # z +- h is exact in fp32
    val = []
    for d in (h, -h):
        g, out = Mat(rows, cols, F32, values=z + d), Mat(rows, cols, F32)
        canz.canz_act_forward([canz.Act(rows=rows, cols=cols, gate=g, out=out, act=kind, dtype=F32)], stream())
        torch.cuda.synchronize()
        val.append(out.get())
    g, one, dg = Mat(rows, cols, F32, values=z), Mat(rows, cols, F32, values=np.ones_like(z)), Mat(rows, cols, F32)
    canz.canz_act_backward([canz.ActGrad(rows=rows, cols=cols, dout=one, gate=g, dgate=dg, act=kind, dtype=F32, in_dtype=F32)], stream())
    torch.cuda.synchronize()
    b, bs = bounds(kind, z)
    b2, _ = bounds(kind, z + h)
    tol = h * h / 6 + (b + b2 + np.abs(z) * 2 ** -23) / h + bs + 2 ** -22
    assert (np.abs(dg.get() - (val[0] - val[1]) / (2 * h)) <= tol).all()


def test_in_place_and_halves_of_one_matrix(canz):
    """gate and up as the halves of one matrix, their gradients over them, out over dout."""
    import torch
    rng = np.random.default_rng(9)
    rows, cols = 50, 333
    gate, up, dout = inputs(rng, rows, cols, BF16)
    both = Mat(rows, 2 * cols, BF16, values=np.concatenate([gate, up], axis=1))
    d = Mat(rows, cols, BF16, values=dout)
    p = both.data_ptr()
    canz.canz_act_backward([canz.ActGrad(rows=rows, cols=cols, dout=d, gate=p, up=p + 2 * cols, dgate=p, dup=p + 2 * cols, out=d, in_dtype=BF16,
                                         ld_in=2 * cols)], stream())
    torch.cuda.synchronize()
    b, bs = bounds(L.SILU, gate)
    want_dg, want_du = L.gated_grad(L.SILU, dout, gate, up)
    want = L.gated(L.SILU, gate, up)
    got = both.get()
    close(got[:, :cols], want_dg, np.abs(dout * up) * bs + np.abs(want_dg) * 2 ** -22 + FLUSH, BF16)
    close(got[:, cols:], want_du, np.abs(dout) * b + np.abs(want_du) * 2 ** -23 + FLUSH, BF16)
    close(d.get(), want, b * np.abs(up) + np.abs(want) * 2 ** -23, BF16)


def test_far_and_non_finite_arguments(canz):
    import torch
    z = np.array([[200.0, -200.0, 88.0, -88.0, 1e30, -1e30, np.nan, 5.0, -0.0, 13.0, -13.0, -40.0]])
    for kind in (L.SILU, L.GELU, L.RELU):
        g, out, one, dg = Mat(1, 12, F32, values=z), Mat(1, 12, F32), Mat(1, 12, F32, values=np.ones((1, 12))), Mat(1, 12, F32)
        canz.canz_act_forward([canz.Act(rows=1, cols=12, gate=g, out=out, act=kind, dtype=F32)], stream())
        canz.canz_act_backward([canz.ActGrad(rows=1, cols=12, dout=one, gate=g, dgate=dg, act=kind, dtype=F32, in_dtype=F32)], stream())
        torch.cuda.synchronize()
        got, d = out.view().cpu().numpy()[0], dg.view().cpu().numpy()[0]
        assert np.isnan(got[6]) and np.isnan(d[6])
        assert got[0] == 200 and got[2] == 88 and got[4] == np.float32(1e30) and abs(got[1]) < 1e-30 and abs(got[3]) < 1e-30 and got[5] == 0 and got[8] == 0
        assert d[0] == 1 and d[4] == 1 and abs(d[1]) < 1e-30 and d[5] == 0
    z = np.array([[np.inf, -np.inf]])
    g, out, one, dg = Mat(1, 2, F32, values=z), Mat(1, 2, F32), Mat(1, 2, F32, values=np.ones((1, 2))), Mat(1, 2, F32)
    canz.canz_act_forward([canz.Act(rows=1, cols=2, gate=g, out=out, act=L.RELU, dtype=F32)], stream())
    canz.canz_act_backward([canz.ActGrad(rows=1, cols=2, dout=one, gate=g, dgate=dg, act=L.RELU, dtype=F32, in_dtype=F32)], stream())
    torch.cuda.synchronize()
    assert out.view().cpu().numpy().tolist() == [[np.inf, 0.0]] and dg.view().cpu().numpy().tolist() == [[1.0, 0.0]]


def test_each_result_alone(canz):
    """Every result by itself has the bits it has among the others; dout is not needed for out."""
    import torch
    rng = np.random.default_rng(10)
    rows, cols = 9, 200
    gate, up, dout = inputs(rng, rows, cols, BF16)
    g, u, d = image_of(gate), image_of(up), Mat(rows, cols, BF16, values=dout)
    full = {k: Mat(rows, cols, BF16) for k in ("dgate", "dup", "out")}
    canz.canz_act_backward([canz.ActGrad(rows=rows, cols=cols, dout=d, gate=g, up=u, **full)], stream())
    torch.cuda.synchronize()
    for k, v in full.items():
        one = Mat(rows, cols, BF16)
        canz.canz_act_backward([canz.ActGrad(rows=rows, cols=cols, dout=None if k == "out" else d, gate=g, up=u, **{k: one})], stream())
        torch.cuda.synchronize()
        assert np.array_equal(one.get(), v.get())
    g, u, g8 = Mat(rows, cols, BF16, values=gate), Mat(rows, cols, BF16, values=up), Image(rows, cols)
    canz.canz_act_forward([canz.Act(rows=rows, cols=cols, gate=g, up=u, gate8=g8)], stream())
    torch.cuda.synchronize()
    same_image(g8, gate)
