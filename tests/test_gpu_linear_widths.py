"""GPU: canz_linear where its kernels change with the columns of C, with an image of the result or with what shares a call: each variant against the fp64 oracle, and its bits against each
other's, which have to be the same since a product alone decides the order of its sums."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, MX8, Mat
from tests.test_gpu_linear import Product, call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("a_dtype", [BF16, MX8])
@pytest.mark.parametrize("m", [1, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("n", [1, 15, 17, 250, 4095, 4096, 4097, 12287, 12288])
def test_few_rows_by_columns(canz, m, n, a_dtype):
    """Without an image (narrow blocks up to 4096 columns), then the same product with one."""
    rng = np.random.default_rng(m * 31 + n)
    k = 1025 if n < 1000 else 300
    p = Product(canz, rng, m, n, k, a_dtype, act=L.GELU, pre=False, exact=False, odd=n % 2 == 1)
    call(canz, [p.group])
    p.check()
    c = p.c.get()
    q = Product(canz, rng, m, n, k, a_dtype)   # an image and another result in one call with it
    fresh = Mat(m, n, p.c.dtype, p.c.ld - n, p.c.shift - 64)
    p.group.c = [fresh]
    call(canz, [q.group, p.group])
    q.check()
    assert np.array_equal(fresh.get(), c)


@pytest.mark.parametrize("n", [100, 4096, 5000])
def test_few_rows_whole_numbers(canz, n):
    """Exact sums, k from less than a unit to many units for each wavefront."""
    rng = np.random.default_rng(n)
    for m in (1, 20, 50):
        for k in (1, 127, 128, 129, 512, 640, 4096, 4200):
            for a_dtype, out in ((BF16, F32), (MX8, BF16)):
                p = Product(canz, rng, m, n, k, a_dtype, out=out, pre=False, sums=False)
                call(canz, [p.group])
                p.check()


def test_one_long_product_among_short_ones(canz):
    """A tile that takes as long as all others of a CU changes the ring of the launch, not a bit of a product."""
    rng = np.random.default_rng(3)
    shapes = [(1000, 1536, 4096), (400, 1536, 256), (2000, 1000, 100), (65, 900, 64)]
    made = [Product(canz, rng, *s, exact=False, pre=False, out=F32) for s in shapes]
    call(canz, [p.group for p in made])
    for p in made:
        p.check()
        fresh = Mat(p.c.rows, p.c.cols, F32)
        p.group.c, c = [fresh], p.c.get()
        call(canz, [p.group])
        assert np.array_equal(fresh.get(), c)
