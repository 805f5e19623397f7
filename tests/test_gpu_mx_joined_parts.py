"""GPU: products whose k is cut into parts that are joined, and products of no k, with alpha, beta and either type of result against the fp64 oracle.
Scales of 1 make products multiples of 1/4 and sums below 36 k < 2^20 for k <= 20000; with alpha 1/2 and beta 2 on whole numbers up to 50 results are
multiples of 1/8 and still exact in fp32; a bf16 result is that rounded once."""
import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests import mx_rules as R
from tests.test_gpu_mx_large_tiles import check, old_result
from tests.test_gpu_mx_product import ULP_BF16, ULP_F32, device, operand, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(65, 100, 16000), (130, 260, 20000), (200, 300, 9001), (513, 400, 7000)])
def test_alpha_beta(canz, m, n, k):
    import torch
    assert R.parts(m, n, k) > 1
    rng = np.random.default_rng(k + 1)
    a, b = operand(rng, m, k), operand(rng, n, k)
    s = MX.product(MX.values(*a), MX.values(*b))
    groups, checks = [], []
    for i, (out_dtype, alpha, beta) in enumerate([(W.DT_F32, 0.5, 2.0), (W.DT_BF16, 0.5, 2.0), (W.DT_F32, -1.0, 0.0), (W.DT_BF16, 1.0, 0.0), (W.DT_BF16, 2.0, -1.0)]):
        c, old = old_result(rng, m, n, out_dtype, n + i)
        if beta == 0.0:
            c[:m, :n] = float("nan")
        groups.append(canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], ldc=n + i, alpha=alpha, beta=beta, out_dtype=out_dtype))
        checks.append((c, m, n, out_dtype, alpha * s + beta * old, old))
    run(canz, groups)                              # five of them in one call, more parts than a launch takes
    for *x, _ in checks:
        check(*x)
    for g, (c, _, _, _, _, old) in zip(groups, checks):
        c[:m, :n] = torch.from_numpy(old).to(c.dtype)
        run(canz, [g])
    for *x, _ in checks:
        check(*x)


@pytest.mark.parametrize("m,n,k", [(65, 100, 16000), (200, 300, 9001)])
def test_rounding_of_alpha_and_beta(canz, m, n, k):
    """Factors that are no powers of two: alpha S rounded (2^-24), the fused sum rounded, rounded to the type."""
    import torch
    rng = np.random.default_rng(k + 2)
    a, b = operand(rng, m, k), operand(rng, n, k)
    s = MX.product(MX.values(*a), MX.values(*b))
    for out_dtype, half in ((W.DT_F32, ULP_F32), (W.DT_BF16, ULP_BF16)):
        c = torch.from_numpy(rng.standard_normal((m, n)).astype(np.float32) * 500).to(torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16).cuda()
        old = c.double().cpu().numpy()
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], alpha=0.3, beta=-0.7, out_dtype=out_dtype)])
        al, be = float(np.float32(0.3)), float(np.float32(-0.7))
        want = al * s + be * old
        first = ULP_F32 * np.abs(al * s)
        bound = first + (ULP_F32 + half) * (np.abs(want) + first) * (1 + 2.0 ** -7)
        assert (np.abs(c.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("m,n", [(1, 70), (3, 129), (200, 33), (1000, 700)])
def test_no_k(canz, m, n):
    """C <- beta C, rounded in fp32 and once more in bf16; exact for a power of two; zeros for beta = 0, whatever was there."""
    import torch
    rng = np.random.default_rng(m)
    for out_dtype, half in ((W.DT_F32, 0.0), (W.DT_BF16, ULP_BF16)):
        for beta in (0.25, -0.7, 1.0, 0.0):
            c = torch.full((m + 1, n + 3), 99.0, dtype=torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16, device="cuda")
            c[:m, :n] = float("nan") if beta == 0.0 else torch.from_numpy(rng.standard_normal((m, n)).astype(np.float32)).cuda().to(c.dtype)
            old = c[:m, :n].double().cpu().numpy()
            run(canz, [canz.MxProduct(m=m, n=n, k=0, c=[c], ldc=n + 3, alpha=3.0, beta=beta, out_dtype=out_dtype)])
            got = c.double().cpu().numpy()
            want = np.zeros((m, n)) if beta == 0.0 else float(np.float32(beta)) * old
            bound = np.zeros((m, n)) if beta in (0.25, 1.0, 0.0) else np.abs(want) * (ULP_F32 + half * (1 + ULP_F32))
            assert (np.abs(got[:m, :n] - want) <= bound).all()
            assert (got[m:] == 99).all() and (got[:, n:] == 99).all()
