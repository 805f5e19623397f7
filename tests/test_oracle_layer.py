"""Pins of oracle/layer.py: hand-worked roundings, closed forms, gradients against differences; and mistakes planted in a copy of its source, each of which a pin has to
catch.  CPU only."""
import inspect
import math
import types

import numpy as np
import pytest

import oracle.layer as L

MODULE = [L]   # the mutation tests put a mutant here


def la():
    return MODULE[0]


def _block(*v):
    x = np.zeros((1, 32))
    x[0, :len(v)] = v
    return x


def pin_grid():
    g = la().GRID
    assert len(g) == 127 and g[0] == 0 and g[1] == 2.0 ** -9 and g[7] == 7 * 2.0 ** -9 and g[8] == 2.0 ** -6 and g[126] == 448
    assert (np.diff(g) > 0).all() and g[0x38] == 1.0 and g[0x3C] == 1.5


def pin_hand_worked_blocks():
    # amax 448: X = 1; 17 and 19 are ties of steps of 2 (codes 16 and 18, 18 and 20), 2^-10 one of the smallest step
    codes, byte = la().encode(_block(448, 17, 19, -17, 18, 16.9, 17.1, 2.0 ** -10, 3 * 2.0 ** -10, 1.0))
    assert byte.tolist() == [[127]]
    assert la().values(codes, byte)[0, :10].tolist() == [448, 16, 20, -16, 18, 16, 18, 0, 2 * 2.0 ** -9, 1.0]
    assert codes[0, :4].tolist() == [0x7E, 0x58, 0x5A, 0xD8]
    # just above 448 X doubles; just above 224 X = 1 still
    assert la().encode(_block(np.nextafter(448, 449)))[1][0, 0] == 128
    assert la().encode(_block(np.nextafter(224, 225)))[1][0, 0] == 127
    assert la().encode(_block(224.0))[1][0, 0] == 126


def pin_limits():
    assert la().encode(_block(0.0))[1][0, 0] == 3 and la().encode(_block(-0.0))[0][0, 0] == 128
    assert la().encode(_block(448 * 2.0 ** -124))[1][0, 0] == 3 and la().encode(_block(449 * 2.0 ** -124))[1][0, 0] == 4
    big = float(np.finfo(np.float32).max)
    codes, byte = la().encode(_block(big, -big, 1.0))
    assert byte[0, 0] == 246 and codes[0, 0] == 0x7E and np.isfinite(la().values(codes, byte).astype(np.float32)).all() and codes[0, 2] == 0
    assert la().encode(_block(448 * 2.0 ** 119))[1][0, 0] == 246 and la().encode(_block(449 * 2.0 ** 118))[1][0, 0] == 246
    for v in (np.inf, -np.inf, np.nan):
        codes, byte = la().encode(np.concatenate([_block(v, 1.0), _block(1.0)], axis=1))
        assert byte[0, 0] == 255 and not codes[0, :32].any()
        got = la().values(codes, byte)
        assert np.isnan(got[0, :32]).all() and got[0, 32] == 1.0


def pin_every_value_is_the_nearest():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((20, 70)) * np.exp2(rng.integers(-140, 120, (20, 1)).astype(float))
    x[3], x[4, 40:] = 0, 0
    codes, byte = la().encode(x)
    assert byte.shape == (20, 3) and codes.shape == (20, 70)
    v = la().values(codes, byte)
    for r in range(20):
        for b in range(3):
            part, got = x[r, 32 * b:32 * b + 32], v[r, 32 * b:32 * b + 32]
            unit = 2.0 ** (int(byte[r, b]) - 127)
            grid = np.concatenate([-L.GRID[::-1], L.GRID]) * unit
            assert np.abs(part).max() <= 448 * unit and (byte[r, b] == 3 or np.abs(part).max() > 224 * unit)
            assert np.array_equal(np.abs(part - got), np.abs(part[:, None] - grid).min(axis=1))
    assert np.array_equal(la().eight(v), v)      # values keep themselves


def pin_layout():
    codes = np.arange(2 * 130, dtype=np.uint64).reshape(2, 130).astype(np.uint8)
    scales = np.arange(10, dtype=np.uint8).reshape(2, 5) + 100
    im = la().pack(codes, scales)
    assert la().image_bytes(2, 130) == im.size == 768 and la().image_bytes(0, 5) == 0 and la().image_bytes(1, 1) == 256
    assert la().image_bytes(1000, 128) == 132096            # 128000 + 4000, to a multiple of 256
    assert im[129] == 129 and im[130] == 0 and im[256] == 130 and im[512] == 100 and im[516] == 104 and im[517] == 0 and im[520] == 105


def pin_bf16():
    x = np.array([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -20, -3.14159, np.inf, 2.0 ** -133, 3e38], np.float32)
    want = [1.0, 1.0, 1 + 2 * 2.0 ** -7, 1 + 2.0 ** -7, -3.140625, np.inf, 2.0 ** -133]
    assert la().round_bf16(x)[:7].tolist() == want and np.isnan(la().round_bf16(np.array([np.nan]))[0])


def pin_activations():
    z = np.array([-3.0, -1.0, 0.0, 0.5, 2.0])
    assert np.allclose(la().act(L.SILU, z), [v / (1 + math.exp(-v)) for v in z], rtol=1e-14)
    # Phi by its series at 1/2 and tables: Phi(1) = .841344746068543, Phi(2) = .977249868051821, Phi(3) = .998650101968370
    assert np.allclose(la().act(L.GELU, np.array([1.0, 2.0, -1.0, -3.0])), [.841344746068543, 2 * .977249868051821, -.158655253931457, -3 * .001349898031630], rtol=1e-12)
    assert la().act(L.RELU, z).tolist() == [0, 0, 0, 0.5, 2] and la().slope(L.RELU, z).tolist() == [0, 0, 0, 1, 1]
    assert la().act(L.NONE, z).tolist() == z.tolist() and la().slope(L.NONE, z).tolist() == [1] * 5
    h = 1e-6
    for kind in (L.SILU, L.GELU):
        diff = (la().act(kind, z + h) - la().act(kind, z - h)) / (2 * h)
        assert np.allclose(la().slope(kind, z), diff, atol=1e-9)
    rng = np.random.default_rng(1)
    dout, gate, up = rng.standard_normal((3, 4, 5))
    for kind in (L.NONE, L.SILU, L.GELU):
        for u in (None, up):
            dg, du = la().gated_grad(kind, dout, gate, u)
            num = (dout * (la().gated(kind, gate + h, u) - la().gated(kind, gate - h, u))) / (2 * h)
            assert np.allclose(dg, num, atol=1e-8)
            if u is None:
                assert du is None
            else:
                assert np.allclose(du, dout * (la().gated(kind, gate, u + h) - la().gated(kind, gate, u - h)) / (2 * h), atol=1e-8)


def pin_norm():
    y, rstd = la().norm(np.array([[3.0, 4.0], [0.0, 0.0]]), np.array([1.0, 2.0]), 0.5)
    assert np.allclose(rstd, [13 ** -0.5, 0.5 ** -0.5]) and np.allclose(y, [[3 / 13 ** 0.5, 8 / 13 ** 0.5], [0, 0]])
    rng = np.random.default_rng(2)
    h, dy, dsum = rng.standard_normal((3, 3, 6))
    w, eps, d = rng.standard_normal(6), 0.1, 1e-6
    loss = lambda h, w: (la().norm(h, w, eps)[0] * dy).sum() + (h * dsum).sum()  # noqa: E731
    dx, dw = la().norm_grad(dy, h, la().norm(h, w, eps)[1], w, dsum)
    for i in range(3):
        for j in range(6):
            e = np.zeros((3, 6))
            e[i, j] = d
            assert abs(dx[i, j] - (loss(h + e, w) - loss(h - e, w)) / (2 * d)) < 1e-8
    for j in range(6):
        e = np.zeros(6)
        e[j] = d
        assert abs(dw[j] - (loss(h, w + e) - loss(h, w - e)) / (2 * d)) < 1e-8
    assert np.allclose(la().norm_grad(dy, h, la().norm(h, w, eps)[1], w)[0], dx - dsum)


def pin_linear():
    a, b = np.array([[1.0, 2.0], [3.0, 4.0]]), np.array([[5.0, 6.0], [-7.0, -8.0], [0.0, 1.0]])
    c, z = la().linear(a, b, 0.5, np.array([1.0, 2.0, 3.0]), L.RELU, 2.0, np.ones((2, 3)))
    assert z.tolist() == [[9.5, -9.5, 4.0], [20.5, -24.5, 5.0]] and c.tolist() == [[11.5, 2.0, 6.0], [22.5, 2.0, 7.0]]
    c, z = la().linear(a, b, r=np.full((2, 3), np.nan))
    assert c.tolist() == z.tolist() == [[17, -23, 2], [39, -53, 4]]


PINS = [v for k, v in list(globals().items()) if k.startswith("pin_")]


@pytest.mark.parametrize("pin", PINS, ids=lambda p: p.__name__)
def test_pin(pin):
    pin()


MUTANTS = [
    ("MIN_EXP, MAX_EXP = -124, 119", "MIN_EXP, MAX_EXP = -125, 119"),
    ("MIN_EXP, MAX_EXP = -124, 119", "MIN_EXP, MAX_EXP = -124, 120"),
    ("MIN_EXP, MAX_EXP = -124, 119", "MIN_EXP, MAX_EXP = -124, 118"),
    ("for m in range(8)][:-1]", "for m in range(8)]"),
    ("for e in range(1, 16)", "for e in range(1, 15)"),
    ("e[amax > 448.0 * 2.0 ** (cand - 1)]", "e[amax >= 448.0 * 2.0 ** (cand - 1)]"),
    ("e[amax > 448.0 * 2.0 ** (cand - 1)]", "e[amax > 480.0 * 2.0 ** (cand - 1)]"),
    ("(below < above) | ((below == above) & (low % 2 == 0))", "(below < above) | ((below == above) & (low % 2 == 1))"),
    ("(below < above) | ((below == above) & (low % 2 == 0))", "below <= above"),
    ("128 * np.signbit(v)", "128 * (v < 0)"),
    ("code = np.where(bad[..., None], 0, code)", "code = np.where(bad[..., None], 1, code)"),
    ("np.where(bad, NAN_BYTE, e + 127)", "e + 127"),
    ("np.where(codes & 128, -1.0, 1.0)", "1.0"),
    ("np.exp2(scales.astype(np.float64) - 127)", "np.exp2(scales.astype(np.float64) - 126)"),
    ("b + 0x7FFF + ((b >> 16) & 1)", "b + 0x8000"),
    ("codes + codes // BLOCK", "codes"),
    ("z / (1 + np.exp(-z))", "z / (1 + np.exp(z))"),
    ("z * 0.5 * _erfc(-z / math.sqrt(2))", "z * 0.5 * _erfc(-z)"),
    ("p + z * p * (1 - p)", "p + z * p"),
    ("(z > 0).astype", "(z >= 0).astype"),
    ("z * np.exp(-z * z / 2)", "z * np.exp(-z * z)"),
    ("a if up is None else a * up", "a"),
    ("(d * up, dout * act(kind, gate))", "(d, dout * act(kind, gate))"),
    ("(d * up, dout * act(kind, gate))", "(d * up, dout * gate)"),
    ("(h * h).mean(axis=1) + eps", "(h * h).mean(axis=1)"),
    ("(h * h).mean(axis=1) + eps", "(h * h).sum(axis=1) + eps"),
    ("h * rstd[:, None] * weight, rstd", "h * rstd[:, None], rstd"),
    ("u - n * (u * n).mean(axis=1, keepdims=True)", "u - n * (dy * n).mean(axis=1, keepdims=True)"),
    ("dx if dsum is None else dx + dsum", "dx"),
    ("(dy * n).sum(axis=0)", "(u * n).sum(axis=0)"),
    ("z if bias is None else z + bias", "z"),
    ("alpha * (a @ b.T)", "a @ b.T"),
    ("c if beta == 0.0 else c + beta * r", "c + beta * r if r is not None else c"),
]


@pytest.mark.parametrize("old,new", MUTANTS)
def test_planted_mistake_is_caught(old, new):
    src = inspect.getsource(L)
    assert src.count(old) == 1
    m = types.ModuleType("oracle.layer_mutant")
    m.__package__ = "oracle"
    exec(compile(src.replace(old, new), L.__file__, "exec"), m.__dict__)
    MODULE[0] = m
    caught = False
    try:
        for pin in PINS:
            try:
                pin()
            except Exception:
                caught = True
                break
    finally:
        MODULE[0] = L
    assert caught
