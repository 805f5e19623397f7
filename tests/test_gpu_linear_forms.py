"""GPU: canz_linear's kernels that may do one and the same product, against each other: C has the same bits whatever the width of a block, the rows that share its launch, or the ring of its stages."""
import numpy as np
import pytest

from oracle import layer as L
from tests import linear_rules as R
from tests.layer_harness import BF16, F32, MX8, Image, Mat
from tests.test_gpu_linear import Product, call

pytestmark = pytest.mark.gpu

LONG_AMONG_SHORT = [(1000, 1536, 4096), (400, 1536, 256), (2000, 1000, 100), (65, 900, 64)]


def test_shapes_reach_their_kernels():
    assert [R.few_width(n, False) for n in (1, 4096, 4097, 12287, 12288)] == [16, 16, 32, 32, 64]
    assert [R.few_width(n, True) for n in (1, 4096, 4097, 12287, 12288)] == [32, 32, 32, 32, 64]
    large, tiles, four = R.one_launch(LONG_AMONG_SHORT)
    assert not large and tiles > R.lib().cus() and four
    large, tiles, four = R.one_launch(LONG_AMONG_SHORT[:1] * 4)
    assert not large and tiles > R.lib().cus() and not four
    assert all(R.one_small_tile_to_a_cu(*s) and R.one_launch([s])[2] for s in LONG_AMONG_SHORT[:2])


@pytest.mark.parametrize("a_dtype", [BF16, MX8])
@pytest.mark.parametrize("m", [1, 16, 17, 33, 64])
@pytest.mark.parametrize("n", [1, 33, 250, 1000, 4096, 4097])
def test_few_rows_with_an_image_of_z(canz, m, n, a_dtype):
    """An image takes wider blocks up to 4096 columns.  C with it and without it, alone and beside a product of more rows, which the launch then has registers for."""
    rng = np.random.default_rng(m * 31 + n)
    k = 1025 if n < 1000 else 300
    p = Product(canz, rng, m, n, k, a_dtype, act=L.SILU, pre=False, sums=False, exact=False, odd=n % 2 == 1)
    call(canz, [p.group])
    p.check()
    c = p.c.get()
    more = Product(canz, rng, 64, n, 256, a_dtype, sums=False)
    for pre in (False, True):
        for company in ([], [more.group]):
            fresh = Mat(m, n, p.c.dtype, p.c.ld - n, p.c.shift - 64)
            p.pre = Image(m, n) if pre else None
            p.group.c, p.group.pre8 = [fresh], [p.pre] if pre else []
            call(canz, company + [p.group])
            assert np.array_equal(fresh.get(), c)
            p.check()
    more.check()


def test_one_product_in_either_ring(canz):
    """Alone and among short ones with four stages, among its like with two."""
    rng = np.random.default_rng(4)
    p = Product(canz, rng, *LONG_AMONG_SHORT[0], exact=False, pre=False, out=F32)
    call(canz, [p.group])
    p.check()
    c = p.c.get()
    like = [Product(canz, rng, *LONG_AMONG_SHORT[0], exact=False, pre=False, out=F32) for _ in range(3)]
    short = [Product(canz, rng, *s, exact=False, pre=False, out=F32) for s in LONG_AMONG_SHORT[1:]]
    for company in (like, short):
        fresh = Mat(p.c.rows, p.c.cols, F32)
        p.group.c = [fresh]
        call(canz, [q.group for q in company] + [p.group])
        assert np.array_equal(fresh.get(), c)
    for q in like + short:
        q.check()
