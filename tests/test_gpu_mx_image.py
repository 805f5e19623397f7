"""GPU: canz_mx_quantize and canz_mx_dequantize against the fp64 oracle, bit for bit: rounding is exact arithmetic followed by one
comparison, so there is no tolerance.  Images lie between guard bytes, matrices have rows further apart than their length."""
import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

GUARD = 256


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def device_matrix(x, dtype, ld, fill=7.0):
    """x (fp32 values) in a buffer of row length ld, `fill` behind every row, one more row of it at the end.  Returns (buffer, values)."""
    import torch
    rows, cols = x.shape
    buf = torch.full((rows + 1, ld), fill, dtype=torch.bfloat16 if dtype == W.DT_BF16 else torch.float32)
    buf[:rows, :cols] = torch.from_numpy(x).to(buf.dtype)
    held = buf[:rows, :cols].float().numpy().astype(np.float64)
    return buf.cuda(), held


class Image:
    """A device image between guard bytes."""

    def __init__(self, canz, rows, cols, fill=0xA5):
        import torch
        self.rows, self.cols, self.n = rows, cols, canz.canz_mx_image_bytes(rows, cols)
        self.buf = torch.full((self.n + 2 * GUARD,), fill, dtype=torch.uint8, device="cuda")
        self.fill = fill

    def data_ptr(self):
        return self.buf.data_ptr() + GUARD

    def host(self):
        b = self.buf.cpu().numpy()
        assert (b[:GUARD] == self.fill).all() and (b[GUARD + self.n:] == self.fill).all(), "bytes around the image were written"
        return b[GUARD:GUARD + self.n]

    def check(self, x, mode, noise=None):
        codes, scales, clean = MX.unpack(self.host(), self.rows, self.cols)
        want_c, want_s = MX.quantize(x, mode, noise)
        assert np.array_equal(scales, want_s)
        bad = np.argwhere(codes != want_c)
        assert len(bad) == 0, "code of %s: %d for %d" % (bad[0], codes[tuple(bad[0])], want_c[tuple(bad[0])])
        assert clean, "the padding is not zero"


def hard_values(rows, cols, seed):
    """Gaussian values with everything a rounding can trip over: ties, borders of the scale rules, zeros of either sign, whole blocks of
    zeros, denormal and largest magnitudes, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    x *= np.exp2(rng.integers(-3, 4, (rows, cols))).astype(np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 4.0, 3.0, 1.0], dtype=np.float32)
    pick = rng.random((rows, cols)) < 0.3
    x[pick] = rng.choice(ties, pick.sum()) * rng.choice([-1, 1], pick.sum())
    x[rng.random((rows, cols)) < 0.1] = 0.0
    x[rng.random((rows, cols)) < 0.02] = -0.0
    blocks = [(0.0, 0.0), (1e-38, 1e-45), (3e38, 1e37), (2.0 ** -126, 2.0 ** -149), (2.0 ** 100, 1.0)]
    for r in range(rows):
        if r % 5 == 1:
            big, small = blocks[(r // 5) % len(blocks)]
            x[r] = rng.uniform(-1, 1, cols).astype(np.float32) * np.where(rng.random(cols) < 0.5, big, small).astype(np.float32)
        if r % 5 == 3:
            x[r] *= np.float32(2.0) ** rng.integers(-60, 60)
    special = rng.random((rows, cols)) < 0.002
    x[special] = rng.choice(np.array([np.inf, -np.inf, np.nan], dtype=np.float32), special.sum())
    return x


SHAPES = [(1, 1), (1, 32), (1, 33), (3, 31), (32, 32), (33, 65), (64, 128), (65, 129), (127, 96), (128, 128), (130, 257), (300, 77), (31, 1000),
          (200, 1)]


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_images_bit_for_bit(canz, rows, cols, dtype):
    import torch
    for case, (mode, noisy, sides, pad) in enumerate([(0, False, "both", 0), (1, False, "row", 3), (0, True, "both", 5), (1, True, "col", 1),
                                                      (1, False, "col", 8), (0, True, "row", 0)]):
        mats, noise, held = [], [], []
        for i in range(2):
            buf, h = device_matrix(hard_values(rows, cols, 100 * case + i), dtype, cols + pad)
            mats.append(buf), held.append(h)
            noise.append(np.random.default_rng(case * 7 + i).integers(0, 256, (rows, cols)).astype(np.uint8))
        by_row = [Image(canz, rows, cols) for _ in mats] if sides != "col" else []
        by_col = [Image(canz, cols, rows) for _ in mats] if sides != "row" else []
        u = [torch.from_numpy(n).cuda() for n in noise] if noisy else []
        canz.canz_mx_quantize([canz.MxGroup(rows=rows, cols=cols, ld=cols + pad, mat=mats, by_row=by_row, by_col=by_col, noise=u, dtype=dtype)],
                              mode, stream())
        torch.cuda.synchronize()
        for i in range(2):
            n = noise[i] if noisy else None
            if by_row:
                by_row[i].check(held[i], mode, n)
            if by_col:
                by_col[i].check(held[i].T, mode, n.T if noisy else None)


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
def test_every_scale_byte_and_code(canz, dtype):
    """Blocks whose largest magnitude runs over every exponent, with mantissas around the border of the ceil rule."""
    import torch
    rng = np.random.default_rng(3)
    exps = np.arange(-149, 128)
    rows = []
    for e in exps:
        for m in (1.0, 1.25, 1.5, 1.5078125, 1.984375):
            row = rng.uniform(-1, 1, 32) * 2.0 ** e * m
            row[rng.integers(0, 32)] = 2.0 ** e * m
            rows.append(row)
    x = np.array(rows).astype(np.float32)
    buf, held = device_matrix(x, dtype, 32)
    for mode in (0, 1):
        img, img_t = Image(canz, *x.shape), Image(canz, x.shape[1], x.shape[0])
        canz.canz_mx_quantize([canz.MxGroup(rows=x.shape[0], cols=32, mat=[buf], by_row=[img], by_col=[img_t], dtype=dtype)], mode, stream())
        out = torch.full(x.shape, 3.0, device="cuda")
        canz.canz_mx_dequantize([canz.MxGroup(rows=x.shape[0], cols=32, mat=[out], by_row=[img])], stream())
        torch.cuda.synchronize()
        img.check(held, mode)
        img_t.check(held.T, mode)
        want = MX.values(*MX.quantize(held, mode))
        assert np.array_equal(out.cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (33, 65), (64, 128), (65, 129), (128, 40), (300, 77), (31, 1000)])
def test_dequantize_bit_for_bit(canz, rows, cols, dtype):
    """Any codes and scale bytes, through either image; what lies behind the rows stays."""
    import torch
    rng = np.random.default_rng(rows * 1000 + cols)
    for side, pad in (("row", 0), ("col", 0), ("row", 3), ("col", 5)):
        r, c = (rows, cols) if side == "row" else (cols, rows)
        codes = rng.integers(0, 16, (r, c)).astype(np.uint8)
        # 2^-127 .. 2^125 and NaN; 0.5 times 2^-127 is a denormal of bf16 as well
        scales = rng.choice(np.array([0, 1, 2, 100, 120, 127, 130, 200, 252, 255], dtype=np.uint8), (r, -(-c // 32)))
        img = torch.from_numpy(MX.pack(codes, scales)).cuda()
        buf, _ = device_matrix(np.zeros((rows, cols), dtype=np.float32), dtype, cols + pad)
        kw = dict(by_row=[img]) if side == "row" else dict(by_col=[img])
        canz.canz_mx_dequantize([canz.MxGroup(rows=rows, cols=cols, ld=cols + pad, mat=[buf], dtype=dtype, **kw)], stream())
        torch.cuda.synchronize()
        want = MX.values(codes, scales)
        want = want if side == "row" else want.T
        got = buf.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got[:rows, :cols], want, equal_nan=True)
        assert (got[rows] == 7.0).all() and (got[:, cols:] == 7.0).all()


def test_many_matrices_groups_and_empty_ones(canz):
    """More matrices than a launch takes, several groups, some of them empty; each matrix gives what it gives alone."""
    import torch
    rng = np.random.default_rng(11)
    groups, checks = [], []
    for rows, cols, n in ((40, 70, 70), (0, 9, 2), (130, 33, 3), (9, 0, 2), (64, 64, 0)):
        mats, imgs, held = [], [], []
        for i in range(n):
            buf, h = device_matrix(rng.standard_normal((rows, cols)).astype(np.float32), W.DT_F32, max(cols, 1))
            mats.append(buf), held.append(h)
            imgs.append(Image(canz, rows, cols))
        groups.append(canz.MxGroup(rows=rows, cols=cols, ld=max(cols, 1), mat=mats, by_row=imgs))
        checks += [(im, h) for im, h in zip(imgs, held)]
    canz.canz_mx_quantize(groups, MX.CEIL, stream())
    torch.cuda.synchronize()
    for im, h in checks:
        if h.size:
            im.check(h, MX.CEIL)
        else:
            im.host()


def test_noise_is_unbiased(canz):
    """The mean over all 256 bytes is the value to within 1/512 of a step (ceil rule)."""
    import torch
    rng = np.random.default_rng(12)
    row = rng.standard_normal(96).astype(np.float32)
    buf, held = device_matrix(np.tile(row, (256, 1)), W.DT_F32, 96)
    u = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, 96)
    img = Image(canz, 256, 96)
    out = torch.empty(256, 96, device="cuda")
    canz.canz_mx_quantize([canz.MxGroup(rows=256, cols=96, mat=[buf], by_row=[img], noise=[u])], MX.CEIL, stream())
    canz.canz_mx_dequantize([canz.MxGroup(rows=256, cols=96, mat=[out], by_row=[img])], stream())
    mean = out.double().mean(0).cpu().numpy()
    unit = np.repeat(np.exp2(MX.quantize(held[:1], MX.CEIL)[1][0].astype(float) - 127), 32)
    a = np.abs(row) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0)) * unit
    assert (np.abs(mean - row) <= step / 512 * (1 + 1e-6)).all()
    log("noise: largest bias %.3g of a step" % np.max(np.abs(mean - row) / step))


def test_large_matrix_offsets(canz):
    """A matrix whose element offsets pass 2^31: its last rows are what they are alone."""
    import torch
    rows, cols = 66000, 32900                        # 2.17e9 elements, 4.3 GB
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(200, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(torch.bfloat16)
    x[-200:] = tail
    img = torch.empty(canz.canz_mx_image_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    img_t = torch.empty(canz.canz_mx_image_bytes(cols, rows), dtype=torch.uint8, device="cuda")
    canz.canz_mx_quantize([canz.MxGroup(rows=rows, cols=cols, mat=[x], by_row=[img], by_col=[img_t], dtype=canz.DT_BF16)], 0, stream())
    x.zero_()
    for kw, axis in ((dict(by_row=[img]), 1), (dict(by_col=[img_t]), 0)):
        canz.canz_mx_dequantize([canz.MxGroup(rows=rows, cols=cols, mat=[x], dtype=canz.DT_BF16, **kw)], stream())
        torch.cuda.synchronize()
        assert not x[:-300].any()
        got = x[-208:].double().cpu().numpy()
        held = np.zeros((208, cols))
        held[8:] = tail.double().cpu().numpy()
        if axis == 0:                                # 66000 = 32 * 2062 + 16: the blocks along rows are cut at a multiple of 32
            first = (rows - 208) % 32
            want = np.zeros((cols, first + 208))
            want[:, first:] = held.T
            want = MX.values(*MX.quantize(want, 0))[:, first:].T
        else:
            want = MX.values(*MX.quantize(held, 0))
        assert np.array_equal(got, want)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_noise_anywhere(canz, shift):
    """Noise bytes at addresses of any alignment, rows of odd length, and the largest and smallest noise there is."""
    import torch
    rows, cols = 131, 77
    x = hard_values(rows, cols, 40 + shift)
    buf, held = device_matrix(x, W.DT_F32, cols)
    for u in (np.random.default_rng(shift).integers(0, 256, (rows, cols)).astype(np.uint8), np.zeros((rows, cols), np.uint8), np.full((rows, cols), 255, np.uint8)):
        around = torch.full((rows * cols + 8,), 200, dtype=torch.uint8, device="cuda")
        noise = around[shift:shift + rows * cols]
        noise.copy_(torch.from_numpy(u.ravel()))
        assert noise.data_ptr() % 4 == shift
        a, b = Image(canz, rows, cols), Image(canz, cols, rows)
        canz.canz_mx_quantize([canz.MxGroup(rows=rows, cols=cols, mat=[buf], by_row=[a], by_col=[b], noise=[noise])], MX.FLOOR, stream())
        torch.cuda.synchronize()
        a.check(held, MX.FLOOR, u)
        b.check(held.T, MX.FLOOR, u.T)


@pytest.mark.parametrize("dtype", [W.DT_F32, W.DT_BF16])
def test_noise_at_every_scale(canz, dtype):
    """Blocks of every magnitude from denormal to the largest, each with all digits of its type and elements far below the largest, next to blocks of
    very different magnitudes, zeros and NaN."""
    import torch
    rng = np.random.default_rng(61)
    rows = cols = 32 * 9
    exps = rng.permutation(np.arange(81 * 4) % 277 - 149)
    for rep in range(4):
        x = rng.uniform(1.0, 2.0, (rows, cols)) * rng.choice([-1, 1], (rows, cols))
        x *= np.exp2(-rng.integers(0, 13, (rows, cols)).astype(np.float64)) * (rng.random((rows, cols)) < 0.95)
        block = exps[rep * 81:rep * 81 + 81].reshape(9, 9)
        x = (x * np.exp2(np.repeat(np.repeat(block, 32, 0), 32, 1).astype(np.float64))).astype(np.float32)
        x[5, 40] = np.nan
        x[77, 200] = -np.inf
        u = rng.integers(0, 256, (rows, cols)).astype(np.uint8)
        buf, held = device_matrix(x, dtype, cols)
        a, b = Image(canz, rows, cols), Image(canz, cols, rows)
        for mode in (MX.FLOOR, MX.CEIL):
            canz.canz_mx_quantize([canz.MxGroup(rows=rows, cols=cols, mat=[buf], by_row=[a], by_col=[b], noise=[torch.from_numpy(u).cuda()], dtype=dtype)],
                                  mode, stream())
            torch.cuda.synchronize()
            a.check(held, mode, u)
            b.check(held.T, mode, u.T)
