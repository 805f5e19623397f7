"""GPU: 8-bit images that come from elsewhere, with scale bytes that canz_mx_eight_store does not write (it writes 3 .. 246 and 255): every byte with every code, wherever images are read.

A value is the code's times 2^(byte - 127), exact in fp32 but for bytes from 247 on, where it may be an infinity, and rounded once to bf16 (whose spacing below 2^-126 is 2^-133, where bytes 0 to 2 reach further
down).  The codes 127 and 255 are NaN."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, MX8, HALF, Image, Mat, held, stream
from tests.test_gpu_linear import call

pytestmark = pytest.mark.gpu


def every():
    """(codes, scale bytes): row r has byte r in all of its blocks, and every code."""
    return np.tile(np.arange(256, dtype=np.uint8), (256, 1)), np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 8))


def finite(rows):
    """The same with those rows, and without NaN codes."""
    codes, scales = every()
    codes = np.where((codes & 127) == 127, 5, codes).astype(np.uint8)
    return codes[rows], scales[rows]


def as_held(x, dtype):
    with np.errstate(over="ignore"):
        return held(x, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_load(canz, dtype):
    import torch
    codes, scales = every()
    back = Mat(256, 256, dtype)
    canz.canz_mx_eight_load([canz.Mx8Group(rows=256, cols=256, mat=[back], image=[Image(256, 256, codes, scales)], dtype=dtype)], stream())
    torch.cuda.synchronize()
    assert np.array_equal(back.view().double().cpu().numpy(), as_held(L.values(codes, scales), dtype), equal_nan=True)


def test_padding_of_a_short_row(canz):
    """Scale 0 in the padding stands for zeros."""
    import torch
    codes, scales = finite(np.array([0, 1, 127]))
    codes, scales = codes[:, 100:133], scales[:, :2]
    back = Mat(3, 33, F32, 5)
    canz.canz_mx_eight_load([canz.Mx8Group(rows=3, cols=33, ld=back.ld, mat=[back], image=[Image(3, 33, codes, scales)], dtype=F32)], stream())
    torch.cuda.synchronize()
    assert np.array_equal(back.get(), held(L.values(codes, scales), F32))


@pytest.mark.parametrize("m", [4, 100])
def test_operands(canz, m):
    """As A and as B, by few rows and by tiles: C = A (2^60 I) in fp32 is what bf16 holds of A times 2^60; sums of A's rows are those of the values themselves."""
    codes, scales = finite(np.arange(m) % 4)
    scales[0, 1::2] = 130                 # tiny blocks and large ones in a row
    a = L.values(codes, scales)
    eye = np.eye(256) * 2.0 ** 60
    c, s = Mat(m, 256, F32), Mat(1, m, F32)
    call(canz, [canz.Linear(m=m, n=256, k=256, a=[Image(m, 256, codes, scales)], b=[Mat(256, 256, BF16, values=eye)], c=[c], a_sums=[s], a_dtype=MX8, out_dtype=F32)])
    assert np.array_equal(c.get(), held(held(a, BF16) * 2.0 ** 60, F32))
    assert (np.abs(s.get()[0] - a.sum(1)) <= 260 * HALF[F32] * np.abs(a).sum(1) + 260 * 2.0 ** -149).all()
    d = Mat(256, m, F32)
    call(canz, [canz.Linear(m=256, n=m, k=256, a=[Mat(256, 256, BF16, values=eye)], b=[Image(m, 256, codes, scales)], c=[d], b_dtype=MX8, out_dtype=F32)])
    assert np.array_equal(d.get(), held(held(a, BF16) * 2.0 ** 60, F32).T)
    d = Mat(16, m, F32)
    call(canz, [canz.Linear(m=16, n=m, k=256, a=[Mat(16, 256, BF16, values=eye[100:116])], b=[Image(m, 256, codes, scales)], c=[d], b_dtype=MX8, out_dtype=F32)])
    assert np.array_equal(d.get(), held(held(a, BF16) * 2.0 ** 60, F32).T[100:116])


def test_arguments_of_gradients(canz):
    """An activation's and a norm's backward pass from an image whose blocks are of byte 0."""
    import torch
    codes, scales = finite(np.zeros(3, int))
    h = L.values(codes, scales)
    ones = Mat(3, 256, F32, values=np.ones((3, 256)))
    out = Mat(3, 256, F32)
    canz.canz_act_backward([canz.ActGrad(rows=3, cols=256, gate=Image(3, 256, codes, scales), out=out, act=L.NONE, dtype=F32, in_dtype=MX8)], stream())
    torch.cuda.synchronize()
    assert np.array_equal(out.get(), held(h, F32))
    rstd, w, dw = np.full(3, 2.0 ** 100), np.ones((1, 256)), Mat(1, 256, F32)
    g = [canz.NormGrad(rows=3, cols=256, dy=ones, h=Image(3, 256, codes, scales), rstd=Mat(1, 3, F32, values=rstd[None]), weight=Mat(1, 256, F32, values=w), dweight=dw, dtype=F32,
                       h_dtype=MX8)]
    need = canz.canz_norm_backward_workspace_bytes(g)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    canz.canz_norm_backward(g, ws, need, stream())
    torch.cuda.synchronize()
    want = (h * 2.0 ** 100).sum(0)       # three equal terms of 4 significant bits: exact
    assert np.array_equal(dw.get()[0], want)
