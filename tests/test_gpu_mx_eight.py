"""GPU: canz_mx_eight_store and canz_mx_eight_load against the oracle, bit for bit, padding and guards included."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, Image, Mat, held, same_image, spread, stream

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 31), (3, 32), (5, 33), (7, 127), (2, 128), (9, 129), (33, 1000), (65, 1531), (4, 2048), (3, 5000), (1025, 40)]


def store(canz, mats, images, dtype):
    import torch
    m = mats[0]
    canz.canz_mx_eight_store([canz.Mx8Group(rows=m.rows, cols=m.cols, ld=m.ld, mat=mats, image=images, dtype=dtype)], stream())
    torch.cuda.synchronize()


def load(canz, mats, images, dtype):
    import torch
    m = mats[0]
    canz.canz_mx_eight_load([canz.Mx8Group(rows=m.rows, cols=m.cols, ld=m.ld, mat=mats, image=images, dtype=dtype)], stream())
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_store_and_load(canz, rows, cols, dtype):
    rng = np.random.default_rng(rows * 10007 + cols)
    for pad, shift in ((0, 0), (3, 1)):
        x = [held(spread(rng, rows, cols, -150, 110), dtype) for _ in range(2)]
        x[0][rng.random((rows, cols)) < 0.1] = 0.0
        x[1][0, 0] = -0.0
        mats = [Mat(rows, cols, dtype, pad, shift, v) for v in x]
        images = [Image(rows, cols) for _ in x]
        store(canz, mats, images, dtype)
        for v, im in zip(x, images):
            same_image(im, v)
        back = [Mat(rows, cols, dtype, pad + 2, shift) for _ in x]
        load(canz, back, images, dtype)
        for v, b in zip(x, back):
            assert np.array_equal(b.get(), L.eight(v))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_bf16_value(canz, dtype):
    """Each one in a block of its own (every scale), and 32 neighbours to a block (every code)."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    v = bits.view(np.float32).astype(np.float64)
    for x in (v.reshape(65536, 1), v.reshape(2048, 32)):
        m, im = Mat(*x.shape, dtype, values=x), Image(*x.shape)
        store(canz, [m], [im], dtype)
        same_image(im, x)


def test_borders_of_codes_and_scales(canz):
    """fp32 values at the borders between codes, one step below and above, at scales of both ends, and around 448 X."""
    border = ((L.GRID[1:] + L.GRID[:-1]) / 2).astype(np.float32)
    for unit in (2.0 ** -124, 2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 118):
        rows = []
        for b in (border, np.nextafter(border, np.float32(0)), np.nextafter(border, np.float32(1e9)), L.GRID.astype(np.float32)):
            b = np.resize(b, 4 * 31)
            for part in b.reshape(4, 31):
                rows.append(np.append(part.astype(np.float64), -448.0) * unit)
        for top in (448.0, np.nextafter(np.float32(448), np.float32(449)), 449.0, 224.0, np.nextafter(np.float32(224), np.float32(225))):
            rows.append(np.append(np.linspace(0.0, 3.0, 31).astype(np.float32).astype(np.float64), float(top)) * unit)
        x = held(np.array(rows), F32)
        m, im = Mat(*x.shape, F32, values=x), Image(*x.shape)
        store(canz, [m], [im], F32)
        same_image(im, x)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nan(canz, dtype):
    rng = np.random.default_rng(5)
    x = held(rng.standard_normal((40, 100)), dtype)
    for i, v in enumerate((np.inf, -np.inf, np.nan)):
        x[i, 7 + 32 * i] = v
    x[3, 99], x[4, 96] = np.inf, float(np.finfo(np.float32).max)
    x[4] = held(x[4], dtype) if dtype == F32 else np.where(x[4] > 3.3e38, 3.3895313892515355e38, x[4])
    x[5, :32] = np.nan
    m, im, back = Mat(40, 100, dtype, values=x), Image(40, 100), Mat(40, 100, dtype)
    store(canz, [m], [im], dtype)
    same_image(im, x)
    load(canz, [back], [im], dtype)
    got, want = back.view().double().cpu().numpy(), L.eight(x)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[0, :32]).all() and np.isfinite(got[0, 32:]).all()


def test_load_of_any_codes(canz):
    rng = np.random.default_rng(6)
    codes = rng.integers(0, 256, (300, 200)).astype(np.uint8)
    codes[(codes & 127) == 127] = 5
    scales = rng.integers(3, 247, (300, 7)).astype(np.uint8)
    scales[::50, 2] = 255
    want = L.values(codes, scales)
    for dtype in (F32, BF16):
        back = Mat(300, 200, dtype, 1, 1)
        load(canz, [back], [Image(300, 200, codes, scales)], dtype)
        assert np.array_equal(back.view().double().cpu().numpy(), want, equal_nan=True)


def test_groups_of_different_shapes_and_nothing(canz):
    import torch
    rng = np.random.default_rng(7)
    shapes = [(5, 77), (0, 10), (130, 256), (10, 0), (1, 4097)]
    groups, kept = [], []
    for r, c in shapes:
        if r * c == 0:
            groups.append(canz.Mx8Group(rows=r, cols=c, n_mats=2))
            continue
        x = held(rng.standard_normal((r, c)), BF16)
        m, im = Mat(r, c, BF16, values=x), Image(r, c)
        kept.append((x, m, im))
        groups.append(canz.Mx8Group(rows=r, cols=c, mat=[m], image=[im], dtype=BF16))
    canz.canz_mx_eight_store(groups, stream())
    torch.cuda.synchronize()
    for x, _, im in kept:
        same_image(im, x)


def test_offsets_past_32_bits(canz):
    """A matrix of more than 2^32 bytes and an image of more than 2^31, rows far apart: first, middle and last rows."""
    import torch
    rows, cols, ld = 70000, 32768, 33000
    mat = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    mat.view(rows, ld)[:, :cols].normal_(generator=g)
    im = torch.empty(canz.canz_mx_eight_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    canz.canz_mx_eight_store([canz.Mx8Group(rows=rows, cols=cols, ld=ld, mat=[mat], image=[im], dtype=BF16)], stream())
    back = torch.empty(rows * cols, dtype=torch.bfloat16, device="cuda")
    canz.canz_mx_eight_load([canz.Mx8Group(rows=rows, cols=cols, mat=[back], image=[im], dtype=BF16)], stream())
    torch.cuda.synchronize()
    for r in (0, 1, 32767, 65535, 65536, 69998, 69999):
        x = mat.view(rows, ld)[r:r + 1, :cols].double().cpu().numpy()
        codes, scales = L.encode(x)
        assert np.array_equal(im[r * cols:(r + 1) * cols].cpu().numpy(), codes[0])
        at = rows * cols + r * (cols // 32)
        assert np.array_equal(im[at:at + cols // 32].cpu().numpy(), scales[0])
        assert np.array_equal(back.view(rows, cols)[r].double().cpu().numpy(), L.values(codes, scales)[0])
