"""GPU: canz_norm_forward and canz_norm_backward against the fp64 oracle.

Bounds, in units of U = 2^-24.  A row's sum is added up by threads with at most cols / 512 + 32 elements each, then over the threads in at most 6 + 16 steps: it is off by at
most K U, K = cols / 512 + 64, of the sum of the magnitudes.  rstd is the square root of that: (K / 2 + 6) U of itself; y = h rstd w two roundings more.  In dx = dsum + rstd (u - n mean(u n)) n is
off by one rounding more than rstd, u by one, the mean by (K + 4) U of mean |u n|; the difference, the product and the sum add a rounding each, counted twice here.  dw adds up
rows / groups products in one thread and then at most 64 sums.  Each result is rounded once to its type."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, MX8, U, Image, Mat, close, held, image_of, same_image, stream

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 7), (5, 64), (9, 511), (2, 513), (4, 2048), (3, 2049), (2, 4097), (3, 8193), (2, 16384), (2, 16385), (1, 40000), (1300, 33), (700, 520), (530, 2100)]
EPS = 1e-5


def terms(cols):
    return cols / 512 + 64


def inputs(rng, rows, cols, dtype, sum_dtype):
    x = held(rng.standard_normal((rows, cols)), dtype)
    r = held(rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, 1)).astype(float)), sum_dtype)
    return x, r


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,sum_dtype,weight_dtype", [(BF16, BF16, F32), (BF16, F32, BF16), (F32, F32, F32), (F32, BF16, F32)])
def test_forward(canz, rows, cols, dtype, sum_dtype, weight_dtype):
    import torch
    rng = np.random.default_rng(rows * 1009 + cols)
    x, r = inputs(rng, rows, cols, dtype, sum_dtype)
    w = held(1 + 0.3 * rng.standard_normal((1, cols)), weight_dtype)
    for residual in (True, False):
        h = held((x.astype(np.float32) + r.astype(np.float32)) if residual else x, sum_dtype)      # one rounding to fp32, one to the type
        xm, wm, y, s = Mat(rows, cols, dtype, 3, 1, x), Mat(1, cols, weight_dtype, 0, 1, w), Mat(rows, cols, dtype, 5, 1), Mat(rows, cols, sum_dtype, 1, 1)
        rm = Mat(rows, cols, sum_dtype, 1, 3, r) if residual else None
        rstd, y8 = Mat(1, rows, F32, 0, 1), Image(rows, cols)
        canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=xm, residual=rm, weight=wm, sum=s, y=y, y8=y8, rstd=rstd, dtype=dtype, sum_dtype=sum_dtype,
                                          weight_dtype=weight_dtype, eps=EPS, ldx=xm.ld, lds=s.ld, ldy=y.ld)], stream())
        torch.cuda.synchronize()
        want, want_rstd = L.norm(h, w[0], float(np.float32(EPS)))
        assert np.array_equal(s.get(), h)
        rel = (terms(cols) / 2 + 6) * U
        close(rstd.get()[0], want_rstd, want_rstd * rel, F32, "rstd")
        rel = (terms(cols) / 2 + 9) * U
        close(y.get(), want, np.abs(want) * rel, dtype, "y")
        if dtype == F32:
            same_image(y8, y.get())          # y itself is what was rounded
        else:
            codes, scales = y8.get()
            low, high = (L.encode(want * f)[1] for f in (1 - rel, 1 + rel))
            assert ((scales == low) | (scales == high)).all()
            unit = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)[:, :cols]
            assert (np.abs(L.values(codes, scales) - want) <= np.maximum(np.abs(want) * 2.0 ** -4, unit * 2.0 ** -10) * (1 + 2 * rel) + np.abs(want) * rel).all()


def backward(canz, rows, cols, dtype, sum_dtype, h_dtype, weight_dtype, rng, beta=0.0, dsum=True):
    import torch
    x, r = inputs(rng, rows, cols, dtype, sum_dtype)
    h = held(x + r, min(h_dtype, BF16))
    w, dy = held(1 + 0.3 * rng.standard_normal((1, cols)), weight_dtype), held(rng.standard_normal((rows, cols)), dtype)
    rstd = held(L.norm(h, w[0], EPS)[1], F32)
    h = L.eight(h) if h_dtype == MX8 else h
    ds = held(rng.standard_normal((rows, cols)), sum_dtype) if dsum else None
    old = held(rng.standard_normal((1, cols)), F32)
    hm = image_of(h) if h_dtype == MX8 else Mat(rows, cols, h_dtype, 3, 1, h)
    dx, dw = Mat(rows, cols, sum_dtype, 3, 3), Mat(1, cols, F32, 0, 1, old if beta else np.full((1, cols), np.inf))
    a = canz.NormGrad(rows=rows, cols=cols, dy=Mat(rows, cols, dtype, 1, 1, dy), h=hm, rstd=Mat(1, rows, F32, 0, 3, rstd[None]), weight=Mat(1, cols, weight_dtype, 0, 1, w),
                      dsum=Mat(rows, cols, sum_dtype, 3, 1, ds) if dsum else None, dx=dx, dweight=dw, dtype=dtype, sum_dtype=sum_dtype, h_dtype=h_dtype,
                      weight_dtype=weight_dtype, beta=beta, ldy=cols + 1, lds=cols + 3)
    ws = torch.full((canz.canz_norm_backward_workspace_bytes([a]),), 0xFF, dtype=torch.uint8, device="cuda")
    canz.canz_norm_backward([a], ws, ws.numel(), stream())
    torch.cuda.synchronize()
    want_dx, want_dw = L.norm_grad(dy, h, rstd, w[0], ds)
    n, u = h * rstd[:, None], w * dy
    k = terms(cols)
    part = rstd[:, None] * (np.abs(u) * 8 + np.abs(n) * np.abs(u * n).mean(1, keepdims=True) * (k + 12)) * U
    close(dx.get(), want_dx, part + np.abs(want_dx) * 2 * U, sum_dtype, "dx")
    mag = np.abs(dy * n).sum(0)
    want_dw = want_dw + beta * old[0]
    close(dw.get()[0], want_dw, (mag * (rows / min(rows, 128) + 70) + np.abs(beta * old[0]) * 2) * U, F32, "dw")
    return a, ws


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,sum_dtype,h_dtype,weight_dtype", [(BF16, BF16, BF16, F32), (BF16, F32, F32, BF16), (F32, F32, F32, F32), (BF16, F32, MX8, F32),
                                                                  (BF16, BF16, MX8, BF16), (F32, BF16, F32, F32), (F32, F32, BF16, F32)])
def test_backward(canz, rows, cols, dtype, sum_dtype, h_dtype, weight_dtype):
    rng = np.random.default_rng(rows * 1013 + cols)
    backward(canz, rows, cols, dtype, sum_dtype, h_dtype, weight_dtype, rng)
    backward(canz, rows, cols, dtype, sum_dtype, h_dtype, weight_dtype, rng, beta=0.5, dsum=False)


@pytest.mark.parametrize("cols", [100, 3000, 20000])
def test_in_place_and_one_result_alone(canz, cols):
    """sum over residual, dx over dsum; dx and dweight by themselves have the bits they have together."""
    import torch
    rows = 37
    rng = np.random.default_rng(cols)
    x, r = inputs(rng, rows, cols, BF16, F32)
    w = held(1 + 0.3 * rng.standard_normal((1, cols)), F32)
    xm, rm, wm = Mat(rows, cols, BF16, values=x), Mat(rows, cols, F32, values=r), Mat(1, cols, F32, values=w)
    y, s, y2 = Mat(rows, cols, BF16), Mat(rows, cols, F32), Mat(rows, cols, BF16)
    canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=xm, residual=rm, weight=wm, sum=s, y=y, sum_dtype=F32)], stream())
    canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=xm, residual=rm, weight=wm, y=y2, sum_dtype=F32)], stream())
    torch.cuda.synchronize()
    assert np.array_equal(y.get(), y2.get())
    canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=xm, residual=rm, weight=wm, sum=rm, y=y2, sum_dtype=F32)], stream())
    torch.cuda.synchronize()
    assert np.array_equal(rm.get(), s.get()) and np.array_equal(y.get(), y2.get())
    a, ws = backward(canz, rows, cols, BF16, F32, F32, F32, rng)
    dx, dw = a.dx.get(), a.dweight.get()
    a.dx, a.dweight = None, Mat(1, cols, F32)
    canz.canz_norm_backward([a], ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert np.array_equal(a.dweight.get(), dw)
    a.dx, a.dweight = a.dsum, None
    canz.canz_norm_backward([a], 0, 0, stream())
    torch.cuda.synchronize()
    assert np.array_equal(a.dsum.get(), dx)


def test_gradient_against_differences(canz):
    """Along a direction d: (f(h + t d) - f(h - t d)) / 2t for f = sum dy y(h), from the kernel's own y in fp32.  With t = 2^-7 and |d| of the order of |h| / 8 the third-order
    term is below t^2 |f'''| / 6, a few 1e-4 of sum |dy||y|; the roundings of y count |y| K U / t."""
    import torch
    rng = np.random.default_rng(11)
    rows, cols, t = 6, 700, 2.0 ** -7
    h, d = held(rng.standard_normal((rows, cols)), BF16), held(rng.choice([-0.125, 0.125], (rows, cols)), BF16)
    w, dy = held(1 + 0.3 * rng.standard_normal((1, cols)), F32), held(rng.standard_normal((rows, cols)), F32)
    f, wm, rstd = [], Mat(1, cols, F32, values=w), Mat(1, rows, F32)
    for sign in (1, -1, 0):
        y = Mat(rows, cols, F32)
        canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=Mat(rows, cols, F32, values=h + sign * t * d), weight=wm, y=y, rstd=rstd, dtype=F32, eps=EPS)], stream())
        torch.cuda.synchronize()
        f.append(y.get())
    dx, dw = Mat(rows, cols, F32), Mat(1, cols, F32)
    a = canz.NormGrad(rows=rows, cols=cols, dy=Mat(rows, cols, F32, values=dy), h=Mat(rows, cols, F32, values=h), rstd=rstd, weight=wm, dx=dx, dweight=dw, dtype=F32)
    ws = torch.empty(canz.canz_norm_backward_workspace_bytes([a]), dtype=torch.uint8, device="cuda")
    canz.canz_norm_backward([a], ws, ws.numel(), stream())
    torch.cuda.synchronize()
    diff = (dy * (f[0] - f[1])).sum(1) / (2 * t)
    size = np.abs(dy * f[2]).sum(1)
    assert (np.abs((dx.get() * d).sum(1) - diff) <= size * (t * t + terms(cols) * U / t)).all()
    assert np.allclose((dw.get()[0] * w[0]).sum(), (dy * f[2]).sum(), atol=size.sum() * 100 * U)       # y is linear in w


def test_zero_rows_and_non_finite(canz):
    import torch
    rng = np.random.default_rng(12)
    rows, cols = 6, 300
    x = held(rng.standard_normal((rows, cols)), F32)
    x[1], x[2, 5], x[3, 7] = 0, np.nan, np.inf
    w = np.ones((1, cols))
    xm, y, rstd, y8 = Mat(rows, cols, F32, values=x), Mat(rows, cols, F32), Mat(1, rows, F32), Image(rows, cols)
    canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=xm, weight=Mat(1, cols, F32, values=w), y=y, rstd=rstd, y8=y8, dtype=F32, eps=EPS)], stream())
    torch.cuda.synchronize()
    got = y.view().cpu().numpy()
    assert not got[1].any() and abs(rstd.get()[0, 1] * EPS ** 0.5 - 1) < 1e-6
    assert np.isnan(got[2]).all() and np.isnan(got[3, 7]) and not got[3, :7].any()
    good = [0, 1, 4, 5]
    want, _ = L.norm(x[good], w[0], float(np.float32(EPS)))
    close(got[good].astype(float), want, np.abs(want) * 50 * U, F32)
    same_image(y8, got.astype(float))


def test_no_rows(canz):
    import torch
    dw = Mat(1, 50, F32, values=np.arange(50.0)[None])
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    canz.canz_norm_backward([canz.NormGrad(rows=0, cols=50, dweight=dw, beta=2.0)], ws, 256, stream())
    torch.cuda.synchronize()
    assert np.array_equal(dw.get()[0], 2 * np.arange(50.0))
    canz.canz_norm_backward([canz.NormGrad(rows=0, cols=50, dweight=dw)], ws, 256, stream())
    torch.cuda.synchronize()
    assert not dw.get().any()


def test_several_in_one_call(canz):
    """Entries of different shapes, and one shared workspace: the bits of each alone."""
    import torch
    rng = np.random.default_rng(13)
    made = [backward(canz, r, c, BF16, BF16, MX8, F32, rng)[0] for r, c in ((40, 300), (900, 100), (3, 17000), (17, 5000))]
    alone = [(a.dx.get(), a.dweight.get()) for a in made]
    for a in made:
        a.dx, a.dweight = Mat(a.rows, a.cols, BF16, 3, 3), Mat(1, a.cols, F32, 0, 1)
    ws = torch.full((canz.canz_norm_backward_workspace_bytes(made),), 0xFF, dtype=torch.uint8, device="cuda")
    canz.canz_norm_backward(made, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    for a, (dx, dw) in zip(made, alone):
        assert np.array_equal(a.dx.get(), dx) and np.array_equal(a.dweight.get(), dw)
