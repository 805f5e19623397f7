"""GPU: every form of the kernel of canz_mx_product for up to 64 rows (rows of A 16, 32 or 64 at a time, as images or rounded on the way, over
the three ways to go over B) against the fp64 oracle, on n that end inside a unit of B and k that take every wavefront round its ring
more than once and leave a part of a unit at the end.

Scales within 2^-2 .. 1 (k = 5000) or of 1 (k = 9001) make products multiples of 2^-6 (1/4) and sums below 36 k, less than 2^24 of them: fp32 results are exact, bf16
ones that rounded once.  A matrix with such values is its own rounding, whatever of them a block holds (asserted on the oracle)."""
import functools

import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests import mx_rules as R
from tests.test_gpu_mx_product import device, operand, run, to_bf16

pytestmark = pytest.mark.gpu

# (n, k) on either side of the lines at 4096 and 12288
NARROW, MIDDLE, WIDE = [(333, 9001), (4090, 5000)], [(4100, 9001), (12280, 5000)], [(12300, 5000)]
ROWS = [1, 16, 17, 32, 33, 64]


@functools.lru_cache(maxsize=1)
def weights(n, k):
    rng = np.random.default_rng(n + k)
    codes, scales = operand(rng, n, k, 2 if k == 5000 else 0)
    return MX.values(codes, scales), device((codes, scales))


def sums_are_exact(k):
    return 36 * k * (64 if k == 5000 else 4) < 2 ** 24


@pytest.mark.parametrize("n,k", NARROW + MIDDLE + WIDE)
def test_exact_sums(canz, n, k):
    import torch
    assert R.width(n) == (R.NARROW if (n, k) in NARROW else R.MIDDLE if (n, k) in MIDDLE else R.WIDE) and sums_are_exact(k)
    vb, b = weights(n, k)
    for m in ROWS:
        rng = np.random.default_rng(m)
        codes, scales = operand(rng, m, k, 2 if k == 5000 else 0)
        va = MX.values(codes, scales)
        assert np.array_equal(MX.values(*MX.quantize(va, MX.FLOOR)), va)
        want = MX.product(va, vb)
        lda = k + 3
        x = torch.full((m, lda), float("nan"))
        x[:, :k] = torch.from_numpy(va.astype(np.float32))
        operands = [(canz.DT_MX, device((codes, scales))), (W.DT_BF16, x.to(torch.bfloat16).cuda()), (W.DT_F32, x.cuda())]
        for i, (a_dtype, a) in enumerate(operands):
            for out_dtype in (W.DT_F32, W.DT_BF16):
                c = torch.full((m + 1, n + i), float("nan"), dtype=torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16, device="cuda")
                run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[a], b=[b], c=[c], lda=lda, ldc=n + i, a_dtype=a_dtype, out_dtype=out_dtype)])
                got = c.double().cpu().numpy()
                assert np.array_equal(got[:m, :n], want if out_dtype == W.DT_F32 else to_bf16(want)), (m, a_dtype, out_dtype)
                assert np.isnan(got[m:]).all() and np.isnan(got[:, n:]).all()


@pytest.mark.parametrize("n,k", [(4090, 5000), (12280, 5000), (12300, 5000)])
def test_old_results_and_rounded_operands(canz, n, k):
    """alpha 1/2 and beta 2 on whole numbers up to 50: sums are multiples of 2^-4 below 36 k, results of 2^-5 below 18 k + 100, less than 2^24 of them.  Then
    operands that do change when they are rounded: the bits of their images, and |error| <= k 2^-23 sum |a b|."""
    import torch
    vb, b = weights(n, k)
    for m in (1, 9, 16, 30, 64):
        rng = np.random.default_rng(100 + m)
        codes, scales = operand(rng, m, k, 0)
        old = rng.integers(-50, 51, (m, n)).astype(np.float64)
        want = 0.5 * MX.product(MX.values(codes, scales), vb) + 2 * old
        assert np.array_equal(want.astype(np.float32).astype(np.float64), want)
        for out_dtype in (W.DT_F32, W.DT_BF16):
            c = torch.from_numpy(old).to(torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16).cuda()
            run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device((codes, scales))], b=[b], c=[c], alpha=0.5, beta=2.0, out_dtype=out_dtype)])
            assert np.array_equal(c.double().cpu().numpy(), want if out_dtype == W.DT_F32 else to_bf16(want))
        for a_dtype, dt in ((W.DT_BF16, torch.bfloat16), (W.DT_F32, torch.float32)):
            x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).to(dt).cuda()
            img = torch.empty(canz.canz_mx_image_bytes(m, k), dtype=torch.uint8, device="cuda")
            canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, mat=[x], by_row=[img], dtype=a_dtype)], MX.CEIL, torch.cuda.current_stream().cuda_stream)
            c, d = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
            run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[img], b=[b], c=[c], out_dtype=W.DT_F32)])
            run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[b], c=[d], a_dtype=a_dtype, a_scale_mode=MX.CEIL, out_dtype=W.DT_F32)])
            assert torch.equal(c, d)
            va = MX.values(*MX.quantize(x.double().cpu().numpy(), MX.CEIL))
            err = np.abs(c.double().cpu().numpy() - MX.product(va, vb))
            assert (err <= k * 2.0 ** -23 * MX.product(np.abs(va), np.abs(vb))).all()


@pytest.mark.parametrize("n,k", [(333, 9001), (4100, 9001), (12300, 5000)])
def test_nan_in_the_last_part_of_k(canz, n, k):
    """A NaN in the last row's last element, where a unit of k is not whole, and a NaN block of B there: that row, that column, no more."""
    import torch
    rng = np.random.default_rng(k)
    codes, scales = operand(rng, n, k, 0)
    scales[n - 1, -1] = 255
    b = device((codes, scales))
    vb = MX.values(codes, scales)
    for m in (1, 16, 31, 64):
        va = MX.values(*operand(rng, m, k, 0))
        va[m - 1, k - 1] = np.nan
        with np.errstate(invalid="ignore"):
            want = MX.product(MX.values(*MX.quantize(va, MX.FLOOR)), vb)
        assert np.isnan(want[m - 1]).all() and np.isnan(want[:, n - 1]).all() and np.isfinite(want[:m - 1, :n - 1]).all()
        for a_dtype, dt in ((W.DT_BF16, torch.bfloat16), (W.DT_F32, torch.float32)):
            x = torch.from_numpy(va.astype(np.float32)).to(dt).cuda()
            c = torch.empty(m, n, device="cuda")
            run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[b], c=[c], a_dtype=a_dtype, out_dtype=W.DT_F32)])
            assert np.array_equal(c.double().cpu().numpy(), want, equal_nan=True)
