"""GPU: canz_mx_product against the fp64 oracle.

Products of two elements are exact in fp32.  Where all scales of a test are equal enough that every partial sum is a multiple of one unit
below 2^24 of it, the sums are exact too and an fp32 result has to be exact; a bf16 result is that rounded once.  Elsewhere a sum of k products
rounds at most k times, each time by at most 2^-23 (the matrix cores may cut instead of rounding) of a partial sum, itself at most the sum of magnitudes:
|error| <= k 2^-23 sum |a b|."""
import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests.gpu_harness import log

pytestmark = pytest.mark.gpu

ULP_BF16 = 2.0 ** -8      # half a step relative to the value
ULP_F32 = 2.0 ** -24


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def operand(rng, rows, k, spread=0):
    """(codes, scales) of an image: scales 2^-spread .. 2^0 around 1."""
    codes = rng.integers(0, 16, (rows, k)).astype(np.uint8)
    scales = (127 - rng.integers(0, spread + 1, (rows, -(-k // 32)))).astype(np.uint8)
    return codes, scales


def device(img):
    import torch
    return torch.from_numpy(MX.pack(*img)).cuda()


def workspace(canz, groups, fill=0xFF):
    """Scratch full of NaN bytes: nothing in it may have to start at zero."""
    import torch
    return torch.full((canz.canz_mx_product_workspace_bytes(groups),), fill, dtype=torch.uint8, device="cuda")


def run(canz, groups, ws=None):
    import torch
    ws = workspace(canz, groups) if ws is None else ws
    canz.canz_mx_product(groups, ws, ws.numel(), stream())
    torch.cuda.synchronize()


def to_bf16(x):
    import torch
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 33, 100), (2, 64, 128), (1, 1000, 4000), (3, 257, 1025), (16, 100, 640), (17, 64, 256), (31, 500, 77),
          (33, 129, 300), (64, 64, 1024), (65, 130, 129), (100, 1, 50), (128, 256, 512), (255, 257, 384), (257, 300, 1000), (500, 700, 2100),
          (1, 5000, 64), (5, 40, 9000), (640, 300, 128)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_exact_sums(canz, m, n, k):
    """Scales within 2^-2 .. 1 on either side: products are multiples of 2^-6 and sums below 36 k < 2^18 for k <= 7281; above that
    the scales are 1 and the unit 1/4.  fp32 results are exact, bf16 ones rounded once."""
    import torch
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    spread = 2 if 36 * k * 64 < 2 ** 24 else 0
    assert 36 * k * (64 if spread else 4) < 2 ** 24
    a, b = operand(rng, m, k, spread), operand(rng, n, k, spread)
    want = MX.product(MX.values(*a), MX.values(*b))
    da, db = device(a), device(b)
    for out_dtype, pad in ((W.DT_F32, 0), (W.DT_BF16, 0), (W.DT_F32, 3), (W.DT_BF16, 5)):
        c = torch.full((m + 1, n + pad), float("nan"), dtype=torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16, device="cuda")
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[da], b=[db], c=[c], ldc=n + pad, out_dtype=out_dtype)])
        got = c.double().cpu().numpy()
        assert np.array_equal(got[:m, :n], want if out_dtype == W.DT_F32 else to_bf16(want))
        assert np.isnan(got[m:]).all() and np.isnan(got[:, n:]).all()


@pytest.mark.parametrize("m,n,k", [(65, 100, 16000), (128, 128, 8192), (200, 300, 9001), (513, 400, 7000)])
def test_long_k_in_parts(canz, m, n, k):
    """Few tiles and a long k: k is cut into parts whose sums are joined.  Products that are multiples of 1/4, so that all sums are exact; alone, accumulating
    on an earlier result, and in one call with products that are not cut."""
    import torch
    assert 36 * k * 4 < 2 ** 24
    rng = np.random.default_rng(k)
    a, b, b2 = operand(rng, m, k), operand(rng, n, k), operand(rng, 2000, k)
    want = MX.product(MX.values(*a), MX.values(*b))
    da, db, db2 = device(a), device(b), device(b2)
    c = torch.full((m, n + 3), float("nan"), device="cuda")
    groups = [canz.MxProduct(m=m, n=n, k=k, a=[da], b=[db], c=[c], ldc=n + 3, out_dtype=W.DT_F32)]
    assert canz.canz_mx_product_workspace_bytes(groups) > 256          # it is cut
    run(canz, groups)
    assert np.array_equal(c.double().cpu().numpy()[:, :n], want) and torch.isnan(c[:, n:]).all()
    old = torch.from_numpy(rng.integers(-50, 50, (m, n)).astype(np.float32)).to(torch.bfloat16).cuda()
    h, e = old.clone(), torch.empty(m, 2000, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[da, da], b=[db, db], c=[h, old], alpha=0.5, beta=2.0),
               canz.MxProduct(m=m, n=2000, k=k, a=[da], b=[db2], c=[e], out_dtype=W.DT_F32)] +
              [canz.MxProduct(m=m, n=n, k=k, a=[da], b=[db], c=[torch.empty(m, n, device="cuda")], out_dtype=W.DT_F32) for _ in range(9)])
    assert torch.equal(h, old)
    assert np.array_equal(e.double().cpu().numpy(), MX.product(MX.values(*a), MX.values(*b2)))


@pytest.mark.parametrize("m,n,k", [(1, 300, 5000), (7, 129, 20000), (40, 70, 3000), (300, 260, 4100), (130, 260, 20000)])
def test_wide_scales(canz, m, n, k):
    import torch
    rng = np.random.default_rng(k)
    a, b = operand(rng, m, k, 40), operand(rng, n, k, 40)
    va, vb = MX.values(*a), MX.values(*b)
    want, mag = MX.product(va, vb), MX.product(np.abs(va), np.abs(vb))
    c = torch.empty(m, n, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], out_dtype=W.DT_F32)])
    err = np.abs(c.double().cpu().numpy() - want)
    bound = k * 2.0 ** -23 * mag
    log("wide scales %d x %d x %d: worst error %.3g of the bound" % (m, n, k, np.max(err / bound)))
    assert (err <= bound).all()


@pytest.mark.parametrize("m,n,k", [(1, 65, 300), (20, 65, 300), (150, 140, 300), (300, 290, 260)])
def test_alpha_beta(canz, m, n, k):
    """C <- alpha A B^T + beta C: with exact sums S the result is off by the rounding of alpha S (2^-24) and of the sum."""
    import torch
    rng = np.random.default_rng(4)
    a, b = operand(rng, m, k, 2), operand(rng, n, k, 2)
    s = MX.product(MX.values(*a), MX.values(*b))
    old = rng.standard_normal((m, n)).astype(np.float32) * 50
    for out_dtype, half in ((W.DT_F32, ULP_F32), (W.DT_BF16, ULP_BF16)):
        for alpha, beta in ((0.3, 0.0), (1.0, 1.0), (-0.7, 0.5)):
            c = torch.from_numpy(old).to(torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16).cuda()
            c0 = c.double().cpu().numpy()
            if beta == 0.0:
                c.fill_(float("nan"))                 # not read
            run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], alpha=alpha, beta=beta, out_dtype=out_dtype)])
            al, be = float(np.float32(alpha)), float(np.float32(beta))
            want = MX.product(MX.values(*a), MX.values(*b), al, be, c0)
            # alpha S rounded, the fused sum rounded, rounded to the type
            bound = ULP_F32 * np.abs(al * s) + (ULP_F32 + half) * (np.abs(want) + ULP_F32 * np.abs(al * s)) * 1.01
            assert (np.abs(c.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("a_dtype", [W.DT_F32, W.DT_BF16])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 1000, 1500), (1, 48, 8200), (4, 130, 333), (16, 64, 2048), (17, 300, 129), (32, 77, 640), (50, 200, 700),
                                   (300, 300, 500)])
def test_matrix_operand_is_rounded_as_quantize_rounds(canz, m, n, k, a_dtype):
    """Bit for bit the product of the image; rows of A further apart than k, the rest of them NaN."""
    import torch
    rng = np.random.default_rng(m + n + k)
    dt = torch.float32 if a_dtype == W.DT_F32 else torch.bfloat16
    lda = k + 3
    x = torch.full((m, lda), float("nan"), dtype=dt)
    x[:, :k] = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32) * 3).to(dt)
    if m > 1:
        x[m // 2, :k] = 0
    x = x.cuda()
    b = device(operand(rng, n, k, 2))
    for mode in (0, 1):
        img = torch.empty(canz.canz_mx_image_bytes(m, k), dtype=torch.uint8, device="cuda")
        canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, ld=lda, mat=[x], by_row=[img], dtype=a_dtype)], mode, stream())
        want, got = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[img], b=[b], c=[want], out_dtype=W.DT_F32)])
        run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[b], c=[got], a_dtype=a_dtype, lda=lda, a_scale_mode=mode, out_dtype=W.DT_F32)])
        assert torch.equal(got, want)
        vx = MX.values(*MX.quantize(x[:, :k].double().cpu().numpy(), mode))
        vb = MX.values(*MX.unpack(b.cpu().numpy(), n, k)[:2])
        ref, mag = MX.product(vx, vb), MX.product(np.abs(vx), np.abs(vb))
        assert (np.abs(got.double().cpu().numpy() - ref) <= k * 2.0 ** -23 * mag).all()


@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_nan_blocks_reach_their_rows_and_columns_only(canz, m):
    import torch
    n, k = 200, 700
    rng = np.random.default_rng(m)
    a, b = operand(rng, m, k, 2), operand(rng, n, k, 2)
    a[1][m - 1, 3] = 255
    b[1][77, 21] = 255
    c = torch.empty(m, n, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[device(a)], b=[device(b)], c=[c], out_dtype=W.DT_F32)])
    va, vb = MX.values(*a), MX.values(*b)
    with np.errstate(invalid="ignore"):
        want = MX.product(va, vb)
    bad = np.zeros((m, n), dtype=bool)
    bad[m - 1], bad[:, 77] = True, True
    got = c.double().cpu().numpy()
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad])
    # an activation that is infinite or NaN, rounded in the call
    x = torch.randn(m, k, device="cuda", generator=torch.Generator("cuda").manual_seed(m))
    x[0, 5], x[m - 1, k - 1] = float("inf"), float("nan")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[device(operand(rng, n, k, 2))], c=[c], a_dtype=W.DT_F32, out_dtype=W.DT_F32)])
    got = c.cpu().numpy()
    hit = np.zeros(m, dtype=bool)
    hit[0], hit[m - 1] = True, True
    assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()


def test_empty_extents(canz):
    import torch
    b = device(operand(np.random.default_rng(0), 70, 64))
    # k = 0: C <- beta C
    for m in (1, 3, 200):
        c = torch.full((m, 70), 8.0, device="cuda")
        run(canz, [canz.MxProduct(m=m, n=70, k=0, c=[c], beta=0.25, out_dtype=W.DT_F32)])
        assert (c == 2.0).all()
        c.fill_(float("nan"))
        run(canz, [canz.MxProduct(m=m, n=70, k=0, c=[c], a_dtype=W.DT_BF16, out_dtype=W.DT_F32)])
        assert (c == 0.0).all()
    # m = 0 or n = 0: nothing
    canz.canz_mx_product([canz.MxProduct(m=0, n=70, k=64, b=[b], a=[0], c=[0], a_dtype=W.DT_BF16),
                          canz.MxProduct(m=4, n=0, k=64, b=[0], a=[0], c=[0])], 0, 0, stream())
    torch.cuda.synchronize()


def test_groups_of_different_rows(canz):
    """Experts: more products than a launch takes, their rows from none to hundreds, one shape class of two; each has the bits it has alone."""
    import torch
    rng = np.random.default_rng(9)
    n, k = 150, 400
    groups, outs = [], []
    for i, m in enumerate([0, 1, 37, 200, 5, 0, 64, 300, 2] * 5):
        x = torch.from_numpy(rng.standard_normal((max(m, 1), k)).astype(np.float32)).to(torch.bfloat16).cuda()
        c = torch.full((max(m, 1), n), float("nan"), dtype=torch.bfloat16, device="cuda")
        groups.append(canz.MxProduct(m=m, n=n, k=k, a=[x], b=[device(operand(rng, n, k, 2))], c=[c], a_dtype=W.DT_BF16))
        outs.append(c)
    two = [torch.empty(33, 90, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    groups.append(canz.MxProduct(m=33, n=90, k=77, a=[device(operand(rng, 33, 77, 2)) for _ in two], b=[device(operand(rng, 90, 77, 2)) for _ in two],
                                 c=two))
    outs += two
    run(canz, groups)
    together = [c.clone() for c in outs]
    for c in outs:
        c.fill_(float("nan"))
    for g in groups:
        run(canz, [g])
    for c, t, g in zip(outs, together, groups):
        if g.m == 0:
            assert torch.isnan(t.float()).all()
        else:
            assert torch.equal(c, t)


def test_linear_layer_training_pass(canz):
    """The operators as they are used together: x and dy rounded both ways (dy with noise), y = x W^T, dx = dy W, dW = dy^T x accumulated on an
    earlier gradient, and a Muon step on dW that leaves the images of the new W.  Against the same in fp64; dW and dx also against
    differences of the scalar <dy, x W^T> along directions that the images hold exactly."""
    import torch
    t, n, k = 300, 256, 512
    rng = np.random.default_rng(21)
    x = torch.from_numpy(rng.standard_normal((t, k)).astype(np.float32)).to(torch.bfloat16).cuda()
    dy = torch.from_numpy(rng.standard_normal((t, n)).astype(np.float32) * 1e-3).to(torch.bfloat16).cuda()
    noise = torch.from_numpy(rng.integers(0, 256, (t, n)).astype(np.uint8)).cuda()
    w = torch.from_numpy(W.gen_param(1, 0, n, k)).cuda()
    dw0 = rng.standard_normal((n, k)).astype(np.float32) * 1e-2
    dw = torch.from_numpy(dw0).cuda()
    image = lambda r, c: torch.empty(canz.canz_mx_image_bytes(r, c), dtype=torch.uint8, device="cuda")
    iw, iwt, ix, ixt, idy, idyt = image(n, k), image(k, n), image(t, k), image(k, t), image(t, n), image(n, t)
    canz.canz_mx_quantize([canz.MxGroup(rows=n, cols=k, mat=[w], by_row=[iw], by_col=[iwt])], MX.FLOOR, stream())
    canz.canz_mx_quantize([canz.MxGroup(rows=t, cols=k, mat=[x], by_row=[ix], by_col=[ixt], dtype=W.DT_BF16)], MX.FLOOR, stream())
    canz.canz_mx_quantize([canz.MxGroup(rows=t, cols=n, mat=[dy], by_row=[idy], by_col=[idyt], noise=[noise], dtype=W.DT_BF16)], MX.CEIL, stream())
    y, dx = torch.empty(t, n, device="cuda"), torch.empty(t, k, device="cuda")
    run(canz, [canz.MxProduct(m=t, n=n, k=k, a=[ix], b=[iw], c=[y], out_dtype=W.DT_F32),
               canz.MxProduct(m=t, n=k, k=n, a=[idy], b=[iwt], c=[dx], out_dtype=W.DT_F32),
               canz.MxProduct(m=n, n=k, k=t, a=[idyt], b=[ixt], c=[dw], beta=1.0, out_dtype=W.DT_F32)])
    h = lambda v: v.double().cpu().numpy()
    q = lambda v, mode, u=None: MX.values(*MX.quantize(v, mode, u))
    hx, hdy, hw, u = h(x), h(dy), h(w), noise.cpu().numpy()
    vx, vxt, vw, vwt = q(hx, 0), q(hx.T, 0), q(hw, 0), q(hw.T, 0)
    vdy, vdyt = q(hdy, 1, u), q(hdy.T, 1, u.T)

    def close(got, a, b, more=0.0):
        mag = MX.product(np.abs(a), np.abs(b))
        want = MX.product(a, b) + more
        assert (np.abs(h(got) - want) <= a.shape[1] * 2.0 ** -23 * mag + ULP_F32 * 2 * np.abs(want)).all()
    close(y, vx, vw)
    close(dx, vdy, vwt)
    close(dw, vdyt, vxt, dw0.astype(np.float64))
    # differences: <dy, (x + d) W^T> - <dy, x W^T> for unit steps d, with operands that both images hold alike
    gx = MX.GRID[rng.integers(0, 8, (t, k))]
    gw = MX.GRID[rng.integers(0, 8, (n, k))] * rng.choice([-1.0, 1.0], (n, k))
    gdy = MX.GRID[rng.integers(0, 8, (t, n))]
    f = lambda xx, ww: float(np.sum(gdy * (xx @ ww.T)))
    dev = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()
    for src, r, c, row, col in ((gx, t, k, ix, ixt), (gw, n, k, iw, iwt), (gdy, t, n, idy, idyt)):
        canz.canz_mx_quantize([canz.MxGroup(rows=r, cols=c, mat=[dev(src)], by_row=[row], by_col=[col])], MX.FLOOR, stream())
        torch.cuda.synchronize()
    dw.zero_()
    run(canz, [canz.MxProduct(m=t, n=k, k=n, a=[idy], b=[iwt], c=[dx], out_dtype=W.DT_F32),
               canz.MxProduct(m=n, n=k, k=t, a=[idyt], b=[ixt], c=[dw], beta=1.0, out_dtype=W.DT_F32)])
    base = f(gx, gw)
    for _ in range(10):
        i, j, o = rng.integers(0, t), rng.integers(0, k), rng.integers(0, n)
        step = gx.copy()
        step[i, j] += 1.0
        assert f(step, gw) - base == h(dx)[i, j]      # all of these are multiples of 1/8 far below 2^53, and the kernels' sums below 2^24 of their unit
        step = gw.copy()
        step[o, j] += 1.0
        assert f(gx, step) - base == h(dw)[o, j]
    # the step on this gradient, and the images of what it leaves
    hp = canz.Hparams()
    new, mom = w.clone(), torch.zeros(n, k, device="cuda")
    g = canz.Group(rows=n, cols=k, grad=[dw], mom=[mom], out=[new], grad_dtype=W.DT_F32, out_dtype=W.DT_F32)
    ws = torch.empty(canz.canz_muon_workspace_bytes([g], hp), dtype=torch.uint8, device="cuda")
    canz.canz_muon_step_images([g], hp, [canz.MxImages(by_row=[iw], by_col=[iwt])], MX.FLOOR, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert not torch.equal(new, w)
    for img, v in ((iw, h(new)), (iwt, h(new).T)):
        codes, scales, clean = MX.unpack(img.cpu().numpy(), *v.shape)
        want = MX.quantize(v, 0)
        assert clean and np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])


@pytest.mark.parametrize("out_dtype", [W.DT_F32, W.DT_BF16])
def test_step_images_are_the_step_and_its_images(canz, out_dtype):
    """Several groups, one of them without images, one of them empty: momentum and parameters have the bits canz_muon_step gives."""
    import torch
    hp = canz.Hparams(weight_decay=0.1)
    shapes = [(256, 512, 2), (300, 77, 1), (64, 64, 1), (40, 40, 0)]
    dt = torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16

    def make():
        groups = []
        for s, (rows, cols, n) in enumerate(shapes):
            g = [torch.from_numpy(W.gen_grad(1, 10 * s + i, rows, cols)[0]).cuda() for i in range(n)]
            p = [torch.from_numpy(W.gen_param(1, 10 * s + i, rows, cols)).to(dt).cuda() for i in range(n)]
            groups.append(canz.Group(rows=rows, cols=cols, grad=g, mom=[torch.zeros(rows, cols, device="cuda") for _ in g], out=p,
                                     grad_dtype=W.DT_F32, out_dtype=out_dtype))
        return groups
    a, b = make(), make()
    ws = torch.empty(canz.canz_muon_workspace_bytes(a, hp), dtype=torch.uint8, device="cuda")
    canz.canz_muon_step(a, hp, ws, ws.numel(), stream())
    images = []
    for rows, cols, n in shapes:
        img = lambda r, c: [torch.empty(canz.canz_mx_image_bytes(r, c), dtype=torch.uint8, device="cuda") for _ in range(n)]
        images.append(canz.MxImages() if rows == 64 else canz.MxImages(by_row=img(rows, cols), by_col=img(cols, rows) if rows == 300 else []))
    canz.canz_muon_step_images(b, hp, images, MX.CEIL, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    for x, y, im in zip(a, b, images):
        for i in range(len(x.out)):
            assert torch.equal(x.out[i], y.out[i]) and torch.equal(x.mom[i], y.mom[i])
            v = y.out[i].double().cpu().numpy()
            for seq, val in ((im.by_row, v), (im.by_col, v.T)):
                if seq:
                    codes, scales, clean = MX.unpack(seq[i].cpu().numpy(), *val.shape)
                    want = MX.quantize(val, MX.CEIL)
                    assert clean and np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])


def test_step_images_from_fragments_in_a_graph(canz):
    """Gradients in two column fragments; the step with images recorded and replayed: after every replay the images are those of the parameters, which have
    the bits of as many eager steps."""
    import torch
    hp = canz.Hparams()
    rows, cols = 256, 512

    def make():
        grads = [torch.from_numpy(W.gen_grad(3, i, rows, cols)[0]).cuda() for i in range(2)]
        frags = [f.contiguous() for g in grads for f in g.chunk(2, dim=1)]
        out = [torch.from_numpy(W.gen_param(3, i, rows, cols)).to(torch.bfloat16).cuda() for i in range(2)]
        return canz.Group(rows=rows, cols=cols, tp=2, grad=frags, mom=[torch.zeros(rows, cols, device="cuda") for _ in out], out=out, grad_dtype=W.DT_F32,
                          out_dtype=W.DT_BF16)
    a, b = make(), make()
    ws = torch.empty(canz.canz_muon_workspace_bytes([a], hp), dtype=torch.uint8, device="cuda")
    ws_b = torch.empty_like(ws)
    img = lambda r, c: [torch.empty(canz.canz_mx_image_bytes(r, c), dtype=torch.uint8, device="cuda") for _ in range(2)]
    images = canz.MxImages(by_row=img(rows, cols), by_col=img(cols, rows))
    call = lambda: canz.canz_muon_step_images([b], hp, [images], MX.FLOOR, ws_b, ws_b.numel(), stream())
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    canz.canz_muon_step([a], hp, ws, ws.numel(), stream())
    for _ in range(3):
        canz.canz_muon_step([a], hp, ws, ws.numel(), stream())
        for t in images.by_row + images.by_col:
            t.fill_(0x55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(a.out[i], b.out[i]) and torch.equal(a.mom[i], b.mom[i])
            v = b.out[i].double().cpu().numpy()
            for t, val in ((images.by_row[i], v), (images.by_col[i], v.T)):
                codes, scales, clean = MX.unpack(t.cpu().numpy(), *val.shape)
                want = MX.quantize(val, MX.FLOOR)
                assert clean and np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])


def test_graph_replays_and_other_streams(canz):
    """Rounding and products of one and of many rows recorded into two graphs with workspaces of their own, replayed with eager work between,
    on inputs that change; and the same on a side stream."""
    import torch
    rng = np.random.default_rng(33)
    k, n = 1500, 300
    b = device(operand(rng, n, k, 2))
    graphs = []
    for m in (1, 200):
        x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
        img, c, c2 = torch.empty(canz.canz_mx_image_bytes(m, k), dtype=torch.uint8, device="cuda"), torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        gs = [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[b], c=[c], a_dtype=W.DT_BF16, out_dtype=W.DT_F32),
              canz.MxProduct(m=m, n=n, k=k, a=[img], b=[b], c=[c2], alpha=2.0, out_dtype=W.DT_F32)]
        ws = workspace(canz, gs)

        def call(x=x, img=img, gs=gs, ws=ws, m=m):
            canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, mat=[x], by_row=[img], dtype=W.DT_BF16)], 0, stream())
            canz.canz_mx_product(gs, ws, ws.numel(), stream())
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append((graph, call, x, c, c2))
    for rep in range(4):
        want = []
        for graph, call, x, c, c2 in graphs:
            x.copy_(torch.from_numpy(rng.standard_normal(x.shape).astype(np.float32)))
            call()
            want.append((c.clone(), c2.clone()))
            c.fill_(float("nan")), c2.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (w1, w2), (_, call, _, c, c2) in zip(want, graphs):
            assert torch.equal(c, w1) and torch.equal(c2, w2) and torch.equal(c2, 2 * c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, call, _, c, c2 in graphs:
            c.fill_(float("nan"))
            call()
    side.synchronize()
    for (w1, w2), (_, _, _, c, c2) in zip(want, graphs):
        assert torch.equal(c, w1) and torch.equal(c2, w2)


def test_large_offsets(canz):
    """Operands and results whose byte offsets pass 2^31 and whose element offsets pass 2^32: only the last columns are looked at."""
    import torch
    m, n, k = 70000, 33000, 256                       # C: 2.3e9 elements in bf16, 4.6 GB
    rng = np.random.default_rng(2)
    a, b = operand(rng, 256, k, 2), operand(rng, 256, k, 2)
    big = lambda rows: torch.zeros(canz.canz_mx_image_bytes(rows, k), dtype=torch.uint8, device="cuda")
    x, y = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    x[-256:] = torch.from_numpy(MX.values(*a)).to(torch.bfloat16).cuda()
    y[-256:] = torch.from_numpy(MX.values(*b)).to(torch.bfloat16).cuda()
    ix, iy = big(m), big(n)
    canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, mat=[x], by_row=[ix], dtype=W.DT_BF16),
                           canz.MxGroup(rows=n, cols=k, mat=[y], by_row=[iy], dtype=W.DT_BF16)], 0, stream())
    c = torch.full((m, n), 5.0, dtype=torch.bfloat16, device="cuda")
    run(canz, [canz.MxProduct(m=m, n=n, k=k, a=[ix], b=[iy], c=[c])])
    assert not c[:-256].any() and not c[:, :-256].any()
    assert np.array_equal(c[-256:, -256:].double().cpu().numpy(), to_bf16(MX.product(MX.values(*a), MX.values(*b))))


def test_longest_k_and_most_rows(canz):
    """The documented limit of an extent, with ones: sums of 4194240 < 2^24 are exact."""
    import torch
    top = 4194240
    ones = lambda r, c: torch.ones(r, c, dtype=torch.bfloat16, device="cuda")
    image = lambda r, c: torch.empty(canz.canz_mx_image_bytes(r, c), dtype=torch.uint8, device="cuda")
    a, b = image(65, top), image(40, top)
    x, y = ones(65, top), ones(40, top)
    x[:, -1] = 2.0
    canz.canz_mx_quantize([canz.MxGroup(rows=65, cols=top, mat=[x], by_row=[a], dtype=W.DT_BF16), canz.MxGroup(rows=40, cols=top, mat=[y], by_row=[b], dtype=W.DT_BF16)],
                          0, stream())
    c, c1 = torch.empty(65, 40, device="cuda"), torch.empty(1, 40, device="cuda")
    run(canz, [canz.MxProduct(m=65, n=40, k=top, a=[a], b=[b], c=[c], out_dtype=W.DT_F32),
               canz.MxProduct(m=1, n=40, k=top, a=[x], b=[b], c=[c1], a_dtype=W.DT_BF16, out_dtype=W.DT_F32)])
    assert (c == top + 1).all() and (c1 == top + 1).all()
    del x, y, a, b
    w, v = image(top, 33), torch.ones(top, 33, dtype=torch.bfloat16, device="cuda")
    v[-1] = 4.0
    t = image(33, top)
    canz.canz_mx_quantize([canz.MxGroup(rows=top, cols=33, mat=[v], by_row=[w], by_col=[t], dtype=W.DT_BF16)], 0, stream())
    row = torch.full((1, top), float("nan"), device="cuda")
    run(canz, [canz.MxProduct(m=1, n=top, k=33, a=[ones(1, 33)], b=[w], c=[row], a_dtype=W.DT_BF16, out_dtype=W.DT_F32)])
    assert (row[0, :-1] == 33).all() and row[0, -1] == 132
    gram = torch.empty(33, 33, device="cuda")
    run(canz, [canz.MxProduct(m=33, n=33, k=top, a=[t], b=[t], c=[gram], out_dtype=W.DT_F32)])
    assert (gram == top - 1 + 16).all()


def test_calls_at_once_on_two_streams(canz):
    """Products that are split, that are not, and of few rows, on two streams at a time with workspaces of their own."""
    import torch
    rng = np.random.default_rng(17)
    jobs = []
    for s in range(2):
        groups = []
        for m, n, k in ((100, 200, 9000), (300, 700, 1000), (9, 500, 3000)):
            x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).cuda()
            groups.append(canz.MxProduct(m=m, n=n, k=k, a=[x], b=[device(operand(rng, n, k, 2))], c=[torch.empty(m, n, device="cuda")], a_dtype=W.DT_F32,
                                         out_dtype=W.DT_F32))
        run(canz, groups)
        jobs.append((groups, [g.c[0].clone() for g in groups], workspace(canz, groups), torch.cuda.Stream()))
    for rep in range(5):
        for groups, _, _, _ in jobs:
            for g in groups:
                g.c[0].fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(3):
            for groups, _, ws, st in jobs:
                canz.canz_mx_product(groups, ws, ws.numel(), st.cuda_stream)
        torch.cuda.synchronize()
        for groups, want, _, _ in jobs:
            for g, w in zip(groups, want):
                assert torch.equal(g.c[0], w)


def test_every_kind_in_one_call(canz):
    """Products of every size class, type and beta in one call, operands shared among them, in a workspace of exactly the bytes asked for between
    guards: each has the bits it has alone, and nothing else is written."""
    import torch
    rng = np.random.default_rng(23)
    kinds = [(1, 40, 500), (9, 40, 500), (16, 4100, 96), (17, 40, 500), (33, 40, 500), (64, 300, 260), (65, 300, 260), (300, 300, 260), (100, 200, 9000),
             (7, 33, 0), (0, 40, 500), (70, 40, 8300), (600, 500, 130)]
    b = {(n, k): device(operand(rng, n, k, 2)) for _, n, k in kinds if k}
    groups, outs = [], []
    for i, (m, n, k) in enumerate(kinds * 3):
        a_dtype = (W.DT_BF16, W.DT_F32, canz.DT_MX)[i // len(kinds)]
        out_dtype, beta = (W.DT_F32, W.DT_BF16)[i % 2], 0.5 * (i % 3)
        dt = torch.float32 if out_dtype == W.DT_F32 else torch.bfloat16
        lda, ldc = k + i % 4, n + i % 5
        if k == 0:
            a = 0
        elif a_dtype == canz.DT_MX:
            a = device(operand(rng, max(m, 1), k, 2))
        else:
            a = torch.from_numpy(rng.standard_normal((max(m, 1), lda)).astype(np.float32)).to(torch.bfloat16 if a_dtype == W.DT_BF16 else torch.float32).cuda()
        c = torch.from_numpy(rng.standard_normal((m + 1, ldc)).astype(np.float32)).to(dt).cuda()
        groups.append(canz.MxProduct(m=m, n=n, k=k, a=[a], b=[b.get((n, k), 0)], c=[c], lda=lda, ldc=ldc, alpha=1.5, beta=beta, a_dtype=a_dtype,
                                     out_dtype=out_dtype))
        outs.append(c)
    before = [c.clone() for c in outs]

    def call(gs):
        need = canz.canz_mx_product_workspace_bytes(gs)
        ws = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
        canz.canz_mx_product(gs, ws.data_ptr() + 256, need, stream())
        torch.cuda.synchronize()
        assert (ws[:256] == 0xFF).all() and (ws[256 + need:] == 0xFF).all()
    call(groups)
    together = [c.clone() for c in outs]
    for c, x in zip(outs, before):
        c.copy_(x)
    for g in groups:
        call([g])
    for c, t, x, g in zip(outs, together, before, groups):
        assert torch.equal(c, t)
        assert torch.equal(c[g.m:], x[g.m:]) and torch.equal(c[:, g.n:], x[:, g.n:])
        if g.m and (g.k or g.beta != 1.0):
            assert not torch.equal(c[:g.m, :g.n], x[:g.m, :g.n])
