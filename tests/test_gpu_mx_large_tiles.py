"""GPU: the 256 x 256 kernels of canz_mx_product, all four of them (fp32 and bf16 results, with and without the old ones), on shapes that the
rule sends there (asserted).  Scales within 2^-2 .. 1 make products multiples of 2^-6 and sums below 36 k < 2^18, alpha is 1/2 and beta 2 on
old results that are whole numbers up to 50: every intermediate value is a multiple of 2^-7 below 36 k + 100 < 2^17 for k <= 3600 and so exact in fp32 (24 bits).  An fp32 result has to be exact,
a bf16 one that rounded once."""
import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests import mx_rules as R
from tests.test_gpu_mx_product import device, operand, run, to_bf16

pytestmark = pytest.mark.gpu

# ragged on every side; 8, 13 and 8 units of k (whole rounds of the ring and not), tiles of one round and of two
SHAPES = [(3201, 3970, 1000), (3969, 3300, 1537), (4001, 8100, 1000)]
MIXED = [(1601, 1985, 1000)] * 4                        # fp32 and bf16, with beta and without
COMPANY = [(130, 260, 8300), (200, 300, 100), (70, 33, 600)]   # k in eight parts, a single unit of k, a corner of a tile
TYPES = [(W.DT_F32, 0.0), (W.DT_BF16, 0.0), (W.DT_F32, 2.0), (W.DT_BF16, 2.0)]


def old_result(rng, m, n, out_dtype, ldc):
    """(device buffer of m + 1 rows of ldc, its first m x n as fp64): whole numbers, 99 around them."""
    import torch
    old = rng.integers(-50, 51, (m, n)).astype(np.float64)
    c = torch.full((m + 1, ldc), 99.0, dtype=torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16)
    c[:m, :n] = torch.from_numpy(old).to(c.dtype)
    return c.cuda(), old


def check(c, m, n, out_dtype, want):
    got = c.double().cpu().numpy()
    assert np.array_equal(got[:m, :n], want if out_dtype == W.DT_F32 else to_bf16(want))
    assert (got[m:] == 99).all() and (got[:, n:] == 99).all()


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_exact_sums(canz, m, n, k):
    assert R.large_tiles([(m, n, k)])
    rng = np.random.default_rng(m)
    a, b = operand(rng, m, k, 2), operand(rng, n, k, 2)
    s = MX.product(MX.values(*a), MX.values(*b))
    da, db = device(a), device(b)
    for (out_dtype, beta), pad in zip(TYPES, (0, 0, 3, 5)):
        c, old = old_result(rng, m, n, out_dtype, n + pad)
        if beta == 0.0:
            c[:m, :n] = float("nan")          # not read
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[da], b=[db], c=[c], ldc=n + pad, alpha=0.5, beta=beta, out_dtype=out_dtype)])
        check(c, m, n, out_dtype, 0.5 * s + beta * old)


def test_types_and_lengths_in_one_call(canz):
    """One launch for each type of result, each with products of other lengths and a part of k beside the long ones."""
    assert R.large_tiles(MIXED + COMPANY) and R.parts(*COMPANY[0]) == 8
    rng = np.random.default_rng(5)
    groups, checks = [], []
    for i, (m, n, k) in enumerate(MIXED + COMPANY):
        out_dtype, beta = TYPES[i % 4]
        spread = 2 if 36 * k * 128 < 2 ** 24 else 0
        assert 36 * k * (128 if spread else 8) < 2 ** 24
        a, b = operand(rng, m, k, spread), operand(rng, n, k, spread)
        c, old = old_result(rng, m, n, out_dtype, n + i)
        groups.append(canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], ldc=n + i, alpha=0.5, beta=beta, out_dtype=out_dtype))
        checks.append((c, m, n, out_dtype, 0.5 * MX.product(MX.values(*a), MX.values(*b)) + beta * old))
    run(canz, groups)
    for x in checks:
        check(*x)


def test_same_bits_from_either_tile(canz):
    """Scales over 2^40, so that sums are rounded and their order shows: products that take small tiles alone and large ones in company have the same bits."""
    import torch
    rng = np.random.default_rng(6)
    big, small = SHAPES[0], [(700, 900, 1000), (300, 260, 4100), (129, 500, 8000)]
    assert R.large_tiles([big] + small) and not any(R.large_tiles([s]) for s in small)
    groups = []
    for i, (m, n, k) in enumerate([big] + small):
        out = torch.float32 if i != 1 else torch.bfloat16
        groups.append(canz.MxProduct(m=m, n=n, k=k, a=[device(operand(rng, m, k, 40))], b=[device(operand(rng, n, k, 40))],
                                     c=[torch.full((m, n), float("nan"), dtype=out, device="cuda")],
                                     out_dtype=W.DT_BF16 if i == 1 else W.DT_F32, alpha=0.7))
    run(canz, groups)
    together = [g.c[0].clone() for g in groups]
    for g, t in zip(groups[1:], together[1:]):
        g.c[0].fill_(float("nan"))
        run(canz, [g])
        assert torch.equal(g.c[0], t) and not torch.isnan(t).any()


def test_nan_blocks(canz):
    """A NaN block of A reaches its row, one of B its column, and nothing else."""
    import torch
    m, n, k = SHAPES[0]
    rng = np.random.default_rng(7)
    a, b = operand(rng, m, k, 2), operand(rng, n, k, 2)
    a[1][m - 1, 31], a[1][1000, 0] = 255, 255
    b[1][n - 1, 7] = 255
    c = torch.empty(m, n, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], out_dtype=W.DT_F32)])
    with np.errstate(invalid="ignore"):
        want = MX.product(MX.values(*a), MX.values(*b))
    assert np.isnan(want[[1000, m - 1]]).all() and np.isnan(want[:, n - 1]).all()
    assert np.array_equal(c.double().cpu().numpy(), want, equal_nan=True)


def test_matrix_operand(canz):
    """A rounded by the call: the bits of the product of its image."""
    import torch
    m, n, k = SHAPES[1]
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.standard_normal((m, k + 3)).astype(np.float32)).cuda()
    img = torch.empty(canz.canz_mx_image_bytes(m, k), dtype=torch.uint8, device="cuda")
    canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, ld=k + 3, mat=[x], by_row=[img])], MX.CEIL, torch.cuda.current_stream().cuda_stream)
    b = device(operand(rng, n, k, 2))
    want, got = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[img], b=[b], c=[want], out_dtype=W.DT_F32)])
    run(canz, [canz.MxProduct(m=m, n=n, k=k, lda=k + 3, a=[x], b=[b], c=[got], a_dtype=W.DT_F32, a_scale_mode=MX.CEIL, out_dtype=W.DT_F32)])
    assert torch.equal(got, want)
