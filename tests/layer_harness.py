"""Helpers of the GPU tests around a linear layer: matrices that lie anywhere inside guarded buffers, images, and rounding bounds.

A rounding to a type is off by at most half a step: HALF[dtype] relative to the value, or TINY[dtype] where it is subnormal."""
import numpy as np

from oracle import layer as L

F32, BF16, MX8 = 0, 1, 3
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133}
U = 2.0 ** -24      # fp32 arithmetic


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def tdtype(dtype):
    import torch
    return torch.float32 if dtype == F32 else torch.bfloat16


def held(x, dtype):
    """fp64 values -> the nearest values of the type, as fp64."""
    x = np.asarray(x, dtype=np.float64).astype(np.float32)
    return x.astype(np.float64) if dtype == F32 else L.round_bf16(x)


class Mat:
    """rows x cols elements `ld` apart, `shift` elements behind a 256-byte border, in a buffer whose other elements are NaN and have to stay."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0, values=None):
        import torch
        self.rows, self.cols, self.ld, self.shift, self.dtype = rows, cols, cols + pad, 64 + shift, dtype
        self.buf = torch.full((64 + shift + rows * self.ld + 64,), float("nan"), dtype=tdtype(dtype), device="cuda")
        if values is not None:
            self.set(values)

    def view(self):
        return self.buf[self.shift:self.shift + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols]

    def set(self, values):
        import torch
        self.view().copy_(torch.from_numpy(np.asarray(values, dtype=np.float64)).to("cuda").float().to(tdtype(self.dtype)))

    def data_ptr(self):
        return self.buf.data_ptr() + self.shift * self.buf.element_size()

    def get(self):
        """Values as fp64, after a look at everything around them."""
        import torch
        rest = self.buf.clone()
        rest[self.shift:self.shift + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = float("nan")
        assert torch.isnan(rest).all(), "written outside of the matrix"
        return self.view().double().cpu().numpy()


class Image:
    """An 8-bit image between guards."""

    def __init__(self, rows, cols, codes=None, scales=None):
        import torch
        self.rows, self.cols, self.bytes = rows, cols, L.image_bytes(rows, cols)
        self.buf = torch.full((256 + self.bytes + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        if codes is not None:
            self.buf[256:256 + self.bytes] = torch.from_numpy(L.pack(codes, scales)).cuda()

    def data_ptr(self):
        return self.buf.data_ptr() + 256

    def get(self):
        """(codes, scale bytes), after a look at padding and guards."""
        pitch = -(-self.cols // L.PITCH) * L.PITCH
        b = self.buf.cpu().numpy()
        n, s = self.rows * pitch, self.rows * (pitch // 32)
        assert (b[:256] == 0xA5).all() and (b[256 + n + s:] == 0xA5).all(), "written outside of the image"
        codes, scales = b[256:256 + n].reshape(self.rows, pitch), b[256 + n:256 + n + s].reshape(self.rows, pitch // 32)
        nb = -(-self.cols // 32)
        assert not codes[:, self.cols:].any() and not scales[:, nb:].any(), "padding is not zero"
        return codes[:, :self.cols], scales[:, :nb]


def image_of(x):
    """The image of the values x, made by the oracle."""
    return Image(*x.shape, *L.encode(x))


def same_image(image, x):
    """Bit for bit the oracle's image of x."""
    codes, scales = image.get()
    want = L.encode(x)
    assert np.array_equal(scales, want[1]), "scales"
    assert np.array_equal(codes, want[0]), "codes"


def close(got, want, bound, dtype, what=""):
    """|got - want| within an fp32 error bound and one rounding to the type."""
    err, tol = np.abs(got - want), bound + HALF[dtype] * (np.abs(want) + bound) + TINY[dtype]
    worst = np.max(np.where(tol > 0, err / tol, 0), initial=0.0)
    assert np.isfinite(got).all() and worst <= 1.0, "%s: %.3g times the bound" % (what, worst)


def spread(rng, rows, cols, lo=-20, hi=20):
    """Values whose rows have magnitudes of their own."""
    return rng.standard_normal((rows, cols)) * np.exp2(rng.integers(lo, hi + 1, (rows, 1)).astype(float))
