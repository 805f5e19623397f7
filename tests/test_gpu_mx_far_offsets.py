"""GPU: images of more than 4 GiB and results of more than 2^32 elements.  All but the far end is zeros."""
import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests.test_gpu_mx_product import operand, run, stream, to_bf16

pytestmark = pytest.mark.gpu

ROWS, K, TAIL = 66000, 131072, 80          # 66048 padded rows: 4.33e9 bytes of codes, then 0.27e9 of scales; the last 128 padded rows hold 80 rows


def small_operand(rng, rows, k):
    """Codes up to 2 in magnitude and scales of 1: products are multiples of 1/4 and sums at most 4 k = 2^19."""
    codes, scales = operand(rng, rows, k)
    return np.where(codes & 7 > 4, codes & 8, codes).astype(np.uint8), scales


def far_image(canz, tail):
    """An image of ROWS x K whose last TAIL rows are `tail`, all others zero."""
    import torch
    n = canz.canz_mx_image_bytes(ROWS, K)
    img = torch.zeros(n, dtype=torch.uint8, device="cuda")
    packed = torch.from_numpy(MX.pack(*tail)).cuda()
    codes, scales = 128 * K // 2, 128 * K // 32
    assert packed.numel() == codes + scales and n > 1 << 32
    padded = (ROWS + 63) // 64 * 64
    assert padded - 128 == ROWS - TAIL
    all_codes = padded * K // 2
    assert all_codes > 1 << 32                 # all scales lie past 32 bits, and the last rows' codes too
    img[all_codes - codes:all_codes] = packed[:codes]
    img[n - scales:] = packed[codes:]
    return img


def test_operands_past_32_bits(canz):
    """As the weights of one, 20 and 60 rows and as either operand of the tiles."""
    import torch
    rng = np.random.default_rng(1)
    tail = small_operand(rng, TAIL, K)
    far, vt = far_image(canz, tail), MX.values(*tail)
    for m in (1, 20, 60, 100):
        a = small_operand(rng, m, K)
        da, want = torch.from_numpy(MX.pack(*a)).cuda(), MX.product(MX.values(*a), vt)
        c = torch.full((m, ROWS), 5.0, device="cuda")
        run(canz, [canz.MxProduct(m=m, n=ROWS, k=K, a=[da], b=[far], c=[c], out_dtype=W.DT_F32)])
        assert not c[:, :-TAIL].any() and np.array_equal(c[:, -TAIL:].double().cpu().numpy(), want)
        if m > 1:
            c = torch.full((ROWS, m), 5.0, device="cuda")
            run(canz, [canz.MxProduct(m=ROWS, n=m, k=K, a=[far], b=[da], c=[c], out_dtype=W.DT_F32)])
            assert not c[:-TAIL].any() and np.array_equal(c[-TAIL:].double().cpu().numpy(), want.T)


def test_rounding_past_32_bits(canz):
    """A matrix of 8.65e9 elements and its two images: what comes back at the far ends."""
    import torch
    x = torch.zeros(ROWS, K, dtype=torch.bfloat16, device="cuda")
    x[-TAIL:] = torch.randn(TAIL, K, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(torch.bfloat16)
    held = x[-TAIL:].double().cpu().numpy()
    image = lambda r, c: torch.full((canz.canz_mx_image_bytes(r, c),), 0x55, dtype=torch.uint8, device="cuda")
    row, col = image(ROWS, K), image(K, ROWS)
    canz.canz_mx_quantize([canz.MxGroup(rows=ROWS, cols=K, mat=[x], by_row=[row], by_col=[col], dtype=W.DT_BF16)], MX.FLOOR, stream())
    first = (ROWS - TAIL) % 32                 # the blocks along the rows are cut at multiples of 32
    assert first == 0
    for kw, want in ((dict(by_row=[row]), MX.values(*MX.quantize(held, MX.FLOOR))), (dict(by_col=[col]), MX.values(*MX.quantize(held.T, MX.FLOOR)).T)):
        x.fill_(7.0)
        canz.canz_mx_dequantize([canz.MxGroup(rows=ROWS, cols=K, mat=[x], dtype=W.DT_BF16, **kw)], stream())
        torch.cuda.synchronize()
        assert not x[:-TAIL].any()
        assert np.array_equal(x[-TAIL:].double().cpu().numpy(), want)


def test_result_past_2_32_elements(canz):
    import torch
    m, n, k = 70000, 66000, 200                # 4.62e9 elements
    rng = np.random.default_rng(2)
    a, b = operand(rng, 200, k, 2), operand(rng, 200, k, 2)
    x, y = torch.zeros(m, k, device="cuda"), torch.zeros(n, k, device="cuda")
    x[-200:], y[-200:] = torch.from_numpy(MX.values(*a).astype(np.float32)).cuda(), torch.from_numpy(MX.values(*b).astype(np.float32)).cuda()
    iy = torch.empty(canz.canz_mx_image_bytes(n, k), dtype=torch.uint8, device="cuda")
    canz.canz_mx_quantize([canz.MxGroup(rows=n, cols=k, mat=[y], by_row=[iy])], MX.FLOOR, stream())
    want = MX.product(MX.values(*a), MX.values(*b))
    c = torch.full((m, n), 5.0, dtype=torch.bfloat16, device="cuda")
    for beta in (0.0, 2.0):
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[iy], c=[c], a_dtype=W.DT_F32, beta=beta)])
        assert not c[:-200].any() and not c[:, :-200].any()
        assert np.array_equal(c[-200:, -200:].double().cpu().numpy(), to_bf16(want if beta == 0.0 else want + 2 * to_bf16(want)))
