"""GPU: canz_linear against the fp64 oracle.

Exact sums: operands of whole numbers up to 3 (exact in bf16 and in an 8-bit image), so that every partial sum of k <= 10^5 products is a whole number below 2^20 and a result in fp32 is exact
whatever the order, with alpha, bias and residual chosen so that the rest is exact, too; a bf16 result is that rounded once, and pre8 is the oracle's image bit for bit.

Elsewhere a sum of k products rounds at most k times, each time by at most 2^-23 (the matrix cores may cut instead of rounding) of a partial sum, itself at most the sum of magnitudes:
|error| <= (k + 4) 2^-23 (|alpha| sum |a b| + |bias|), the 4 for alpha, bias and the joined parts; through an activation, whose slope is at most 1.13, times 1.13, plus the activation's own
bound (test_gpu_act.py)."""
import numpy as np
import pytest

from oracle import layer as L
from tests import linear_rules as R
from tests.layer_harness import BF16, F32, MX8, Image, Mat, close, held, image_of, same_image, stream
from tests.test_gpu_act import bounds

pytestmark = pytest.mark.gpu


def whole(rng, rows, cols):
    return rng.integers(-3, 4, (rows, cols)).astype(float)


def operand(x, dtype, trans, pad=0, shift=0):
    """(buffer, distance of rows) of a logical rows x k matrix as it is stored."""
    s = np.ascontiguousarray(x.T) if trans else x
    if dtype == MX8:
        return image_of(s), s.shape[1]
    m = Mat(*s.shape, BF16, pad, shift, s)
    return m, m.ld


def call(canz, groups, fill=0xFF):
    """Enqueues the products with scratch full of NaN bytes, between guards."""
    import torch
    need = canz.canz_linear_workspace_bytes(groups)
    ws = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
    canz.canz_linear(groups, ws, need, stream())
    torch.cuda.synchronize()
    assert (ws[need:] == fill).all(), "written behind the workspace"


class Product:
    """A product with everything on it, its buffers and what they have to hold."""

    def __init__(self, canz, rng, m, n, k, a_dtype=BF16, b_dtype=BF16, out=F32, a_trans=False, b_trans=False, act=L.NONE, bias=BF16, residual=True, pre=True, sums=True,
                 odd=False, alpha=0.5, beta=2.0, old=False, exact=True):
        p = 1 if odd else 0
        gen = whole if exact else lambda rng, r, c: held(rng.standard_normal((r, c)), BF16)
        self.a, self.b = gen(rng, m, k), gen(rng, n, k)
        if not exact:
            self.a = L.eight(self.a.T).T if a_dtype == MX8 and a_trans else L.eight(self.a) if a_dtype == MX8 else self.a
            self.b = L.eight(self.b.T).T if b_dtype == MX8 and b_trans else L.eight(self.b) if b_dtype == MX8 else self.b
        am, lda = operand(self.a, a_dtype, a_trans, 3 * p, p)
        bm, ldb = operand(self.b, b_dtype, b_trans, 5 * p, p)
        self.bias = whole(rng, 1, n) if bias is not None else None
        self.r = whole(rng, m, n)
        self.alpha, self.beta, self.act, self.out, self.exact = alpha, beta, act, out, exact
        self.c = Mat(m, n, out, 3 * p, p, self.r if old else np.full((m, n), np.nan))
        rm = Mat(m, n, out, 5 * p, 3 * p, self.r) if residual else None
        self.pre = Image(m, n) if pre else None
        self.start = whole(rng, 1, m)
        self.s = Mat(1, m, F32, 0, p, self.start) if sums else None
        self.beta = beta if residual or old else 0.0
        opt = lambda x: [] if x is None else [x]  # noqa: E731
        self.group = canz.Linear(m=m, n=n, k=k, a=[am], b=[bm], c=[self.c], bias=opt(None if bias is None else Mat(1, n, bias, 0, p, self.bias)), residual=opt(rm),
                                 pre8=opt(self.pre), a_sums=opt(self.s), a_dtype=a_dtype, b_dtype=b_dtype, out_dtype=out, bias_dtype=F32 if bias is None else bias,
                                 a_trans=a_trans, b_trans=b_trans, act=act, alpha=alpha, beta=self.beta, lda=lda, ldb=ldb, ldc=self.c.ld, ldr=-1 if rm is None else rm.ld)

    def check(self):
        want, z = L.linear(self.a, self.b, self.alpha, None if self.bias is None else self.bias[0], self.act, self.beta, self.r)
        k = self.a.shape[1]
        sums = self.alpha * self.a.sum(1) + self.beta * self.start[0]
        if self.exact and self.act in (L.NONE, L.RELU):
            assert np.array_equal(self.c.get(), held(want, self.out)), "C"
        else:
            mag = (k + 4) * 2.0 ** -23 * (abs(self.alpha) * (np.abs(self.a) @ np.abs(self.b).T) + (0 if self.bias is None else np.abs(self.bias)))
            mag = 0 * mag if self.exact else mag
            close(self.c.get(), want, 1.13 * mag + bounds(self.act, z)[0] + np.abs(self.beta * self.r) * 2.0 ** -23 + np.abs(want) * 2.0 ** -23, self.out, "C")
        if self.pre is not None:
            if self.exact:
                same_image(self.pre, z)
            else:
                codes, scales = self.pre.get()
                unit = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)[:, :z.shape[1]]
                assert (np.abs(L.values(codes, scales) - z) <= np.maximum(np.abs(z) * 2.0 ** -4, unit * 2.0 ** -10) + 1.1 * mag).all()
        if self.s is not None:
            if self.exact:
                assert np.array_equal(self.s.get()[0], sums), "a_sums"
            else:
                close(self.s.get()[0], sums, (k + 4) * 2.0 ** -24 * (np.abs(self.alpha * self.a).sum(1) + np.abs(self.beta * self.start[0])), F32, "a_sums")


FEW = [(1, 1, 1), (1, 33, 100), (2, 64, 128), (1, 1000, 4000), (16, 100, 640), (17, 64, 256), (31, 500, 77), (33, 129, 300), (64, 64, 1024), (5, 40, 9000), (3, 257, 1025), (64, 300, 129)]
SMALL = [(65, 130, 129), (100, 1, 50), (1, 65, 8), (7, 9, 3), (128, 256, 512), (255, 257, 384), (257, 300, 1000), (500, 700, 1048), (640, 304, 128), (72, 8, 1), (130, 1000, 31)]
LARGE = [(4096, 4096, 64), (2560, 6400, 104), (4090, 4095, 33)]
TWO_TO_A_CU = [(1900, 3999, 100), (2048, 4000, 296)]
QUARTERS = [(4200, 4400, 392), (4097, 4104, 776)]
PARTS = [(65, 100, 16000), (128, 128, 8192), (200, 300, 9001), (513, 400, 7000), (100, 1000, 20000)]
ORIENTATIONS = [(False, False), (False, True), (True, False), (True, True)]


def test_shapes_reach_their_kernels():
    assert all(R.few(m) for m, _, _ in FEW) and not any(R.few(m, *t) for m, _, _ in FEW for t in ORIENTATIONS[1:])
    assert all(R.parts(*s) == 1 and R.one_small_tile_to_a_cu(*s) for s in SMALL)
    assert all(R.parts(*s) == 1 and not R.large_tiles(*s) and not R.one_small_tile_to_a_cu(*s) for s in TWO_TO_A_CU)
    assert all(R.parts(*s) == 1 and R.large_tiles(*s) and not R.quarters(*s) for s in LARGE)
    assert all(R.parts(*s) == 1 and R.quarters(*s) > 0 for s in QUARTERS)
    assert all(R.parts(*s) > 1 for s in PARTS)


@pytest.mark.parametrize("a_dtype", [BF16, MX8])
@pytest.mark.parametrize("m,n,k", FEW)
def test_few_rows(canz, m, n, k, a_dtype):
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    for out, odd, b_dtype in ((F32, False, BF16), (BF16, True, BF16), (BF16, False, MX8)):
        p = Product(canz, rng, m, n, k, a_dtype, b_dtype, out, odd=odd)
        call(canz, [p.group])
        p.check()
    p = Product(canz, rng, m, n, k, a_dtype, act=L.SILU, exact=False, odd=True)
    call(canz, [p.group])
    p.check()


@pytest.mark.parametrize("a_trans,b_trans", ORIENTATIONS)
@pytest.mark.parametrize("m,n,k", SMALL)
def test_small_tiles(canz, m, n, k, a_trans, b_trans):
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    for out, odd, a_dtype, b_dtype in ((F32, False, BF16, BF16), (BF16, True, BF16, BF16), (BF16, False, MX8, BF16), (F32, False, BF16, MX8), (F32, True, MX8, MX8)):
        p = Product(canz, rng, m, n, k, a_dtype, b_dtype, out, a_trans, b_trans, odd=odd)
        call(canz, [p.group])
        p.check()
    p = Product(canz, rng, m, n, k, a_trans=a_trans, b_trans=b_trans, act=L.GELU, exact=False)
    call(canz, [p.group])
    p.check()


@pytest.mark.parametrize("a_trans,b_trans", ORIENTATIONS)
@pytest.mark.parametrize("m,n,k", LARGE + QUARTERS + TWO_TO_A_CU)
def test_large_tiles(canz, m, n, k, a_trans, b_trans):
    rng = np.random.default_rng(m + n + k)
    for out, odd in ((BF16, False), (F32, m % 8 != 0)):
        p = Product(canz, rng, m, n, k, BF16, BF16, out, a_trans, b_trans, odd=odd, act=L.RELU)
        call(canz, [p.group])
        p.check()


@pytest.mark.parametrize("a_trans,b_trans", ORIENTATIONS)
@pytest.mark.parametrize("m,n,k", PARTS)
def test_long_k_in_parts(canz, m, n, k, a_trans, b_trans):
    rng = np.random.default_rng(m + n + k)
    for out, b_dtype, odd in ((F32, BF16, False), (BF16, MX8, True)):
        p = Product(canz, rng, m, n, k, BF16, b_dtype, out, a_trans, b_trans, odd=odd)
        call(canz, [p.group])
        p.check()


@pytest.mark.parametrize("act", [L.NONE, L.SILU, L.GELU, L.RELU])
@pytest.mark.parametrize("m,n,k", [(3, 70, 200), (150, 200, 136), (70, 70, 9000)])
def test_each_part_of_the_epilogue(canz, m, n, k, act):
    """Bias in either type or none, residual, old results or neither, image of z or none."""
    rng = np.random.default_rng(m + act)
    for bias in (None, F32, BF16):
        for residual, old in ((False, False), (True, False), (False, True)):
            p = Product(canz, rng, m, n, k, out=BF16 if residual else F32, act=act, bias=bias, residual=residual, old=old, pre=bias != F32, sums=residual, alpha=-0.25 if old else 1.0)
            call(canz, [p.group])
            p.check()


def test_residual_in_place(canz):
    rng = np.random.default_rng(3)
    for m, n, k in ((5, 100, 300), (200, 333, 100), (100, 100, 6000)):
        p = Product(canz, rng, m, n, k, out=BF16, residual=False, old=True, pre=False)
        p.group.residual, p.group.ldr = [p.c], p.c.ld
        call(canz, [p.group])
        p.check()


@pytest.mark.parametrize("m,n", [(1, 1), (5, 100), (300, 333), (128, 256)])
def test_nothing_along_k(canz, m, n):
    rng = np.random.default_rng(m)
    for t in ORIENTATIONS:
        p = Product(canz, rng, m, n, 0, out=BF16, act=L.RELU, a_trans=t[0], b_trans=t[1], odd=True)
        p.group.a = p.group.b = []
        call(canz, [p.group])
        p.check()


def test_no_rows_or_columns(canz):
    """Nothing of C; a_sums is still there to do where n is 0."""
    import torch
    rng = np.random.default_rng(4)
    a = whole(rng, 40, 300)
    am, s = Mat(40, 300, BF16, values=a), Mat(1, 40, F32)
    call(canz, [canz.Linear(m=0, n=5, k=5, n_prods=2), canz.Linear(m=40, n=0, k=300, a=[am], a_sums=[s], n_prods=1), canz.Linear(m=5, n=5, k=5, n_prods=0)])
    assert np.array_equal(s.get()[0], a.sum(1))
    canz.canz_linear([], 0, 0, 0)
    torch.cuda.synchronize()


def test_experts_in_one_call(canz):
    """Products of different extents, orientations, types and kernels in one call, more of each than a launch takes: the results of each alone, bit for bit."""
    rng = np.random.default_rng(5)
    rows = [0, 1, 37, 400, 5, 128, 0, 1000, 64, 65] + [3, 70] * 18
    made = []
    for i, m in enumerate(rows):
        t = ORIENTATIONS[i % 4]
        made.append(Product(canz, rng, m, 300, 200, MX8 if i % 3 == 1 else BF16, MX8 if i % 5 == 1 else BF16, BF16 if i % 2 else F32, *t, odd=i % 7 == 0, act=L.SILU if i % 2 else L.NONE,
                            exact=False))
    made.append(Product(canz, rng, 100, 200, 9000, exact=False))
    made.append(Product(canz, rng, 50, 60, 0, exact=False))
    call(canz, [p.group for p in made])
    for p in made:
        if p.a.shape[0] == 0:
            continue
        p.check()
        c, pre = p.c.get(), p.pre.get()
        again = Product.__new__(Product)
        again.__dict__.update(p.__dict__)
        fresh, image = Mat(p.c.rows, p.c.cols, p.c.dtype, p.c.ld - p.c.cols, p.c.shift - 64), Image(p.c.rows, p.c.cols)
        p.group.c, p.group.pre8, p.group.a_sums = [fresh], [image], []
        call(canz, [p.group], 0)
        assert np.array_equal(fresh.get(), c) and all(np.array_equal(x, y) for x, y in zip(image.get(), pre))


def test_several_products_of_a_group(canz):
    rng = np.random.default_rng(6)
    made = [Product(canz, rng, 90, 100, 264) for _ in range(20)]
    g = made[0].group
    for name in ("a", "b", "c", "bias", "residual", "pre8", "a_sums"):
        setattr(g, name, [getattr(p.group, name)[0] for p in made])
    call(canz, [g])
    for p in made:
        p.check()


def test_non_finite_operands(canz):
    """A NaN or an infinity reaches its own row or column, whatever the kernel; padding that holds NaN reaches nothing."""
    rng = np.random.default_rng(7)
    for m, n, k in ((5, 70, 300), (200, 150, 131), (100, 100, 6000)):
        for t in ORIENTATIONS:
            p = Product(canz, rng, m, n, k, BF16, BF16, F32, *t, odd=True, residual=False, pre=False, sums=False)
            a, b = p.a.copy(), p.b.copy()
            a[2, k - 1], b[3, 0] = np.nan, np.inf
            p.group.a, p.group.b = [operand(a, BF16, t[0], 3, 1)[0]], [operand(b, BF16, t[1], 5, 1)[0]]
            call(canz, [p.group])
            got = p.c.view().double().cpu().numpy()
            want, _ = L.linear(p.a, p.b, p.alpha, p.bias[0])
            assert np.isnan(got[2]).all() and not np.isfinite(got[:, 3]).any()
            keep = np.ix_([i for i in range(m) if i != 2], [j for j in range(n) if j != 3])
            assert np.array_equal(got[keep], want[keep])
            p = Product(canz, rng, m, n, k, MX8, BF16, F32, *t, residual=False, pre=False, sums=False)
            a = np.ascontiguousarray(p.a.T) if t[0] else p.a.copy()
            a[0, -1] = np.inf                                # its block is NaN
            p.group.a = [image_of(a)]
            call(canz, [p.group])
            got = p.c.view().double().cpu().numpy()
            bad = np.isnan(L.eight(a))
            bad = (bad.T if t[0] else bad).any(1)
            want, _ = L.linear(p.a, p.b, p.alpha, p.bias[0])
            assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad])


def test_shared_operands(canz):
    """One matrix as several operands, the same one twice in a product."""
    import torch
    rng = np.random.default_rng(8)
    x = whole(rng, 120, 120)
    xm, c = Mat(120, 120, BF16, values=x), [Mat(120, 120, F32) for _ in range(4)]
    call(canz, [canz.Linear(m=120, n=120, k=120, a=[xm], b=[xm], c=[c[i]], a_trans=t[0], b_trans=t[1], out_dtype=F32) for i, t in enumerate(ORIENTATIONS)])
    for (ta, tb), got in zip(ORIENTATIONS, c):
        assert np.array_equal(got.get(), (x.T if ta else x) @ (x if tb else x.T))
    torch.cuda.synchronize()
