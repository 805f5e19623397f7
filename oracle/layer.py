"""What lies around a step's matrices, in fp64 numpy: 8-bit images, activations, the root-mean-square norm, a linear layer's products, and their gradients.

A block of 32 consecutive elements of a row shares a scale X = 2^(byte - 127), the smallest one of 2^-124 .. 2^119 with amax <= 448 X (else
the largest); an element is the nearest
of the values GRID (E4M3) with a sign, ties to the even code, times X.  Rounding compares with the grid; it uses none of the exponent arithmetic of the device code."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
PITCH = 128
NAN_BYTE = 255
MIN_EXP, MAX_EXP = -124, 119
# code = 8 exponent + mantissa: subnormals m 2^-9, then (1 + m / 8) 2^(exponent - 7); code 127 is NaN
GRID = np.array([m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])
NONE, SILU, GELU, RELU = 0, 1, 2, 3


def round_bf16(x: np.ndarray) -> np.ndarray:
    """fp32 values to the nearest bf16 value, ties to even, as fp64."""
    b = np.ascontiguousarray(np.asarray(x, dtype=np.float32)).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.nan, r.astype(np.float64))


# ---- 8-bit images ---------------------------------------------------------------------------------------------------------------
def scale_exponents(amax: np.ndarray) -> np.ndarray:
    """Exponent of X for blocks of largest magnitude amax (finite)."""
    e = np.full(amax.shape, MIN_EXP, dtype=np.int64)
    for cand in range(MIN_EXP + 1, MAX_EXP + 1):
        e[amax > 448.0 * 2.0 ** (cand - 1)] = cand
    return e


def nearest_code(a: np.ndarray) -> np.ndarray:
    """Code of the grid value nearest to a >= 0, the even code of two at the same distance; the largest beyond it."""
    up = np.clip(np.searchsorted(GRID, a), 1, len(GRID) - 1)
    low = up - 1
    below, above = a - GRID[low], GRID[up] - a
    return np.where((below < above) | ((below == above) & (low % 2 == 0)), low, up)


def encode(x: np.ndarray):
    """Rows of x in blocks of 32.  Returns (codes [rows, cols] with the sign in bit 7, scale bytes [rows, blocks])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    v = np.pad(x, ((0, 0), (0, nb * BLOCK - cols))).reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[..., None], 0.0, v)
    e = scale_exponents(np.abs(v).max(axis=2, initial=0.0))
    code = nearest_code(np.abs(v) / np.exp2(e.astype(np.float64))[..., None]) + 128 * np.signbit(v)
    code = np.where(bad[..., None], 0, code)
    byte = np.where(bad, NAN_BYTE, e + 127)
    return code.reshape(rows, nb * BLOCK)[:, :cols].astype(np.uint8), byte.astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What an image stands for, in fp64."""
    x = np.where(scales == NAN_BYTE, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = np.append(GRID, np.nan)[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return v * np.repeat(x, BLOCK, axis=1)[:, :codes.shape[1]]


def image_bytes(rows: int, cols: int) -> int:
    codes = rows * (-(-cols // PITCH) * PITCH)
    return -(-(codes + codes // BLOCK) // 256) * 256


def pack(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The bytes of an image: codes row by row, padded to 128, then scales row by row; up to a multiple of 256 bytes that nobody writes (zeros here)."""
    rows, cols = codes.shape
    pitch = -(-cols // PITCH) * PITCH
    c, s = np.zeros((rows, pitch), np.uint8), np.zeros((rows, pitch // BLOCK), np.uint8)
    c[:, :cols], s[:, :scales.shape[1]] = codes, scales
    out = np.zeros(image_bytes(rows, cols), np.uint8)
    out[:c.size], out[c.size:c.size + s.size] = c.reshape(-1), s.reshape(-1)
    return out


def eight(x: np.ndarray) -> np.ndarray:
    """The values that the 8-bit image of x stands for."""
    return values(*encode(x))


# ---- activations ----------------------------------------------------------------------------------------------------------------
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(kind: int, z: np.ndarray) -> np.ndarray:
    if kind == SILU:
        return z / (1 + np.exp(-z))
    if kind == GELU:
        return z * 0.5 * _erfc(-z / math.sqrt(2))
    if kind == RELU:
        return np.maximum(z, 0.0)
    return z


def slope(kind: int, z: np.ndarray) -> np.ndarray:
    if kind == SILU:
        p = 1 / (1 + np.exp(-z))
        return p + z * p * (1 - p)
    if kind == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == RELU:
        return (z > 0).astype(np.float64)
    return np.ones_like(z)


def gated(kind: int, gate: np.ndarray, up: np.ndarray | None) -> np.ndarray:
    a = act(kind, gate)
    return a if up is None else a * up


def gated_grad(kind: int, dout: np.ndarray, gate: np.ndarray, up: np.ndarray | None):
    """(dgate, dup)"""
    d = dout * slope(kind, gate)
    return (d, None) if up is None else (d * up, dout * act(kind, gate))


# ---- norm -----------------------------------------------------------------------------------------------------------------------
def norm(h: np.ndarray, weight: np.ndarray, eps: float):
    """(y, rstd)"""
    rstd = 1 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * rstd[:, None] * weight, rstd


def norm_grad(dy: np.ndarray, h: np.ndarray, rstd: np.ndarray, weight: np.ndarray, dsum: np.ndarray | None = None):
    """(dx, dweight)"""
    n, u = h * rstd[:, None], weight * dy
    dx = rstd[:, None] * (u - n * (u * n).mean(axis=1, keepdims=True))
    return dx if dsum is None else dx + dsum, (dy * n).sum(axis=0)


# ---- products -------------------------------------------------------------------------------------------------------------------
def linear(a: np.ndarray, b: np.ndarray, alpha: float = 1.0, bias: np.ndarray | None = None, kind: int = NONE, beta: float = 0.0,
           r: np.ndarray | None = None):
    """(C, z) of act(z) + beta R with z = alpha A B^T + bias; A is m x k and B n x k."""
    z = alpha * (a @ b.T)
    z = z if bias is None else z + bias
    c = act(kind, z)
    return (c if beta == 0.0 else c + beta * r), z
