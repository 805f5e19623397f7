"""GPU: canz_linear, canz_act_* and canz_norm_* where offsets pass 32 bits: rows far apart, matrices of more than 4 GiB, results of more than 2^32 elements; and operands of subnormal values."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, held, stream

pytestmark = pytest.mark.gpu


def call(canz, groups):
    import torch
    ws = torch.empty(canz.canz_linear_workspace_bytes(groups), dtype=torch.uint8, device="cuda")
    canz.canz_linear(groups, ws, ws.numel(), stream())
    torch.cuda.synchronize()


def rows_apart(x, ld):
    """x in rows `ld` apart, NaN around them."""
    import torch
    buf = torch.full((x.shape[0] * ld,), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf.view(x.shape[0], ld)[:, :x.shape[1]] = torch.from_numpy(x).cuda().to(torch.bfloat16)
    return buf


@pytest.mark.parametrize("ld", [4194240, 4194248, 16777216 + 8, 9000001])
@pytest.mark.parametrize("m", [40, 300])
def test_rows_far_apart(canz, m, ld):
    """Along the limit of what the tile kernels take where it lies, above it, and at odd distances; A along and across k, C too."""
    import torch
    rng = np.random.default_rng(m)
    n, k = 72, 200
    a, b = rng.integers(-3, 4, (m, k)).astype(float), rng.integers(-3, 4, (n, k)).astype(float)
    want = a @ b.T
    bm = torch.from_numpy(b).cuda().to(torch.bfloat16)
    c = torch.full((m * ld,), float("nan"), dtype=torch.bfloat16, device="cuda")
    call(canz, [canz.Linear(m=m, n=n, k=k, a=[rows_apart(a, ld)], b=[bm], c=[c], lda=ld, ldc=ld)])
    got = c.view(m, ld)
    assert np.array_equal(got[:, :n].double().cpu().numpy(), held(want, BF16)) and torch.isnan(got[:, n:n + 64]).all()
    del c, got
    c = torch.empty(m, n, device="cuda")
    at = np.ascontiguousarray(a.T)
    call(canz, [canz.Linear(m=m, n=n, k=k, a=[rows_apart(at, ld)], b=[bm], c=[c], lda=ld, a_trans=True, out_dtype=F32)])
    assert np.array_equal(c.double().cpu().numpy(), want)


def test_result_of_more_than_2_32_elements(canz):
    """C of 66000 x 66000 bf16 (8.7 GB): rows at the beginning, the middle and the end."""
    import torch
    m = n = 66000
    k = 64
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b = (torch.randint(-3, 4, (m, k), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    c = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    call(canz, [canz.Linear(m=m, n=n, k=k, a=[a], b=[b], c=[c])])
    bv = b.double().cpu().numpy()
    for r in (0, 1, 32767, 65000, 65535, 65536, 65999):
        assert np.array_equal(c[r].double().cpu().numpy(), held(a[r].double().cpu().numpy()[None] @ bv.T, BF16)[0])


def test_elementwise_past_4_gib(canz):
    """70000 x 32768 bf16 (4.6 GB) through an activation and a norm: rows on both sides of every 32-bit border."""
    import torch
    rows, cols = 70000, 32768
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y = torch.empty_like(x)
    look = (0, 1, 32767, 32768, 65535, 65536, 69999)
    canz.canz_act_forward([canz.Act(rows=rows, cols=cols, gate=x, out=y, act=L.RELU)], stream())
    torch.cuda.synchronize()
    for r in look:
        assert torch.equal(y[r], x[r].clamp(min=0))
    w, rstd = torch.ones(cols, device="cuda"), torch.empty(rows, device="cuda")
    canz.canz_norm_forward([canz.Norm(rows=rows, cols=cols, x=x, weight=w, y=y, rstd=rstd, eps=0.0)], stream())
    torch.cuda.synchronize()
    for r in look:
        want, s = L.norm(x[r:r + 1].double().cpu().numpy(), np.ones(cols), 0.0)
        assert abs(rstd[r].item() / s[0] - 1) < 200 * 2.0 ** -24
        assert (np.abs(y[r].double().cpu().numpy() - want[0]) <= np.abs(want[0]) * (2.0 ** -8 + 2.0 ** -15)).all()


@pytest.mark.parametrize("m", [5, 200])
def test_subnormal_operands(canz, m):
    """bf16 below 2^-126 counts with its value: 3 2^-130 times 2^20 is exact in fp32."""
    import torch
    k, n = 64, 80
    a = torch.full((m, k), 3 * 2.0 ** -130, dtype=torch.bfloat16, device="cuda")
    b = torch.full((n, k), 2.0 ** 20, dtype=torch.bfloat16, device="cuda")
    c = torch.empty(m, n, device="cuda")
    call(canz, [canz.Linear(m=m, n=n, k=k, a=[a], b=[b], c=[c], out_dtype=F32)])
    assert (c.double().cpu().numpy() == 64 * 3 * 2.0 ** -110).all()


def test_largest_matrices(canz):
    """2^34 elements: two results without products (k = 0) in one call, more blocks than a launch has, then an activation over one of them."""
    import torch
    n = 131072
    c = [torch.empty(n, n, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bias = [torch.arange(n, device="cuda").remainder(251).float() - s for s in (100, 120)]
    call(canz, [canz.Linear(m=n, n=n, k=0, a=[0, 0], b=[0, 0], c=c, bias=bias, act=L.NONE)])
    rows = (0, 1, 32767, 65535, 65536, n - 1)
    for x, v in zip(c, bias):
        assert all(torch.equal(x[r].float(), v) for r in rows)
    canz.canz_act_forward([canz.Act(rows=n, cols=n, gate=c[0], out=c[1], act=L.RELU)], stream())
    torch.cuda.synchronize()
    assert all(torch.equal(c[1][r].float(), bias[0].clamp(min=0)) for r in rows)
