"""Microscaled 4-bit images and their products, in fp64 numpy.

A block of 32 consecutive elements of a row shares a scale X = 2^(byte - 127); an element is a code of 4 bits, a sign and one of
GRID, times X.  Rounding here compares with the grid; it uses none of the exponent arithmetic of the device code."""
from __future__ import annotations

import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FLOOR, CEIL = 0, 1
NAN_BYTE = 255
MIN_EXP, MAX_EXP = -127, 125


def scale_exponents(amax: np.ndarray, mode: int) -> np.ndarray:
    """Exponent of X for blocks of largest magnitude amax (finite)."""
    e = np.full(amax.shape, MIN_EXP, dtype=np.int64)
    for cand in range(MIN_EXP + 1, MAX_EXP + 1):
        x = 2.0 ** cand
        # floor: the largest X with 4 X <= amax; ceil: the smallest with 6 X >= amax
        take = amax >= 4.0 * x if mode == FLOOR else amax > 6.0 * (x / 2)
        e[take] = cand
    return e


def nearest_code(a: np.ndarray) -> np.ndarray:
    """Code of the grid value nearest to a >= 0, the even code of two at the same distance."""
    dist = np.abs(a[..., None] - GRID)
    best = dist.min(axis=-1, keepdims=True)
    tied = dist == best
    even = tied & (np.arange(8) % 2 == 0)
    return np.where(tied.sum(-1) == 2, even.argmax(-1), tied.argmax(-1))


def noisy_code(a: np.ndarray, u: np.ndarray) -> np.ndarray:
    """Code of a >= 0 with noise bytes u: one of the two grid values around a, the upper one if its share of the
    distance, in 256ths, reaches 256 with u added."""
    low = np.searchsorted(GRID, a, side="right") - 1
    top = low == 7
    up = np.minimum(low + 1, 7)
    width = np.where(top, 1.0, GRID[up] - GRID[low])
    share = np.round(np.where(top, 0.0, (a - GRID[low]) / width) * 256)    # numpy rounds halves to even
    return np.where(~top & (share + u >= 256), up, low)


def quantize(x: np.ndarray, mode: int = FLOOR, noise: np.ndarray | None = None):
    """Rows of x in blocks of 32.  Returns (codes [rows, cols] with the sign in bit 3, scale bytes [rows, blocks])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    pad = ((0, 0), (0, nb * BLOCK - cols))
    v = np.pad(x, pad).reshape(rows, nb, BLOCK)
    u = None if noise is None else np.pad(noise.astype(np.int64), pad).reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[..., None], 0.0, v)
    e = scale_exponents(np.abs(v).max(axis=2, initial=0.0), mode)
    a = np.abs(v) / np.exp2(e.astype(np.float64))[..., None]
    code = nearest_code(a) if u is None else noisy_code(a, u)
    code = code + 8 * np.signbit(v)
    byte = np.where(bad, NAN_BYTE, e + 127)
    return code.reshape(rows, nb * BLOCK)[:, :cols].astype(np.uint8), byte.astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What an image stands for, in fp64."""
    rows, cols = codes.shape
    x = np.where(scales == NAN_BYTE, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(x, BLOCK, axis=1)[:, :cols]


def image_bytes(rows: int, cols: int) -> int:
    r, k = -(-rows // 64) * 64, -(-cols // 128) * 128
    return r * k // 2 + r * k // 32


def unpack(image: np.ndarray, rows: int, cols: int):
    """(codes, scales, everything else is zero) of an image's bytes: units of 16 rows x 128 columns of codes and of 64 x 128 of scales; two
    units of codes share 32 rows, four rows of one, then four of the other."""
    r, k = -(-rows // 64) * 64, -(-cols // 128) * 128
    n = r * k // 2
    # codes: [32 rows][unit][k unit][block][piece of four rows][row][byte]
    c = image[:n].reshape(r // 32, 2, k // 128, 4, 4, 4, 16).transpose(0, 4, 1, 5, 2, 3, 6).reshape(r, k // 2)
    codes = np.stack([c & 15, c >> 4], axis=-1).reshape(r, k)
    # scales: [64 rows][k unit][block][piece][row][32 rows][unit]
    s = image[n:].reshape(r // 64, k // 128, 4, 4, 4, 2, 2).transpose(0, 5, 3, 6, 4, 1, 2).reshape(r, k // 32)
    nb = -(-cols // BLOCK)
    clean = not codes[rows:].any() and not codes[:, cols:].any() and not s[rows:].any() and not s[:, nb:].any()
    return codes[:rows, :cols], s[:rows, :nb], clean


def pack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The bytes of an image, the inverse of unpack."""
    rows, cols = codes.shape
    r, k = -(-rows // 64) * 64, -(-cols // 128) * 128
    c = np.zeros((r, k), dtype=np.uint8)
    c[:rows, :cols] = codes
    s = np.zeros((r, k // 32), dtype=np.uint8)
    s[:rows, :scales.shape[1]] = scales
    c = (c[:, 0::2] | c[:, 1::2] << 4).reshape(r // 32, 4, 2, 4, k // 128, 4, 16).transpose(0, 2, 4, 5, 1, 3, 6)
    s = s.reshape(r // 64, 2, 4, 2, 4, k // 128, 4).transpose(0, 5, 6, 2, 4, 1, 3)
    return np.concatenate([c.reshape(-1), s.reshape(-1)])


def product(a: np.ndarray, b: np.ndarray, alpha: float = 1.0, beta: float = 0.0, c: np.ndarray | None = None) -> np.ndarray:
    """alpha A B^T + beta C of the values of two images."""
    r = alpha * (a @ b.T)
    return r if beta == 0.0 else r + beta * c
