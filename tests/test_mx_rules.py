"""The shapes of the GPU tests of single kernels of canz_mx_product reach those kernels by the library's own rules, and a product is
treated alike on either side of a line that is not crossed.  CPU only."""
from tests import mx_rules as R
from tests import test_gpu_mx_large_tiles as L


def test_large_tiles_are_reached():
    for s in L.SHAPES:
        assert R.large_tiles([s])
    assert R.large_tiles(L.MIXED + L.COMPANY) and not R.large_tiles(L.COMPANY)


def test_rules_at_their_lines():
    assert [R.width(n) for n in (1, 4095, 4096, 12287, 12288)] == [R.NARROW, R.NARROW, R.MIDDLE, R.MIDDLE, R.WIDE]
    assert R.rounds_on_the_way(16, 1 << 13, 1 << 13) and not R.rounds_on_the_way(16, 1 << 13, (1 << 13) + 1)
    assert not R.rounds_on_the_way(17, 1, 1) and R.rounds_on_the_way(1, 0, 0)
    assert R.parts(64, 1000, 1 << 20) == 1 and R.parts(65, 1000, 20000) == 8 and R.parts(65, 0, 20000) == 1
