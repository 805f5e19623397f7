"""Pins of oracle/mx.py: hand-worked roundings, closed forms, the definition by brute force, the layout; and mistakes planted in a copy
of its source, each of which a pin has to catch.  CPU only."""
import inspect
import math
import types

import numpy as np
import pytest

import oracle.mx as MX

MODULE = [MX]   # the mutation tests put a mutant here


def mx():
    return MODULE[0]


def _block(*v):
    x = np.zeros((1, 32))
    x[0, :len(v)] = v
    return x


def pin_hand_worked_blocks():
    # amax 6: both rules take X = 1; ties go to the even code
    codes, byte = mx().quantize(_block(6, 5, -5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.26, 0.24), MX.FLOOR)
    assert byte.tolist() == [[127]]
    assert codes[0, :11].tolist() == [7, 6, 14, 6, 4, 4, 2, 2, 0, 9, 0]
    # amax 7: the floor rule saturates, the ceil rule doubles X
    codes, byte = mx().quantize(_block(7, 3, -7), MX.FLOOR)
    assert byte[0, 0] == 127 and codes[0, :3].tolist() == [7, 5, 15]
    codes, byte = mx().quantize(_block(7, 3, -7), MX.CEIL)
    assert byte[0, 0] == 128 and codes[0, :3].tolist() == [6, 3, 14]   # 3.5 -> 4, 1.5, -4
    # just above 6 and exactly 6 under the ceil rule
    assert mx().quantize(_block(np.nextafter(6, 7)), MX.CEIL)[1][0, 0] == 128
    assert mx().quantize(_block(6.0), MX.CEIL)[1][0, 0] == 127
    # just below 4 and exactly 4 under the floor rule
    assert mx().quantize(_block(np.nextafter(4, 3)), MX.FLOOR)[1][0, 0] == 126
    assert mx().quantize(_block(4.0), MX.FLOOR)[1][0, 0] == 127


def pin_limits():
    assert mx().quantize(_block(0.0), MX.FLOOR)[1][0, 0] == 0
    assert mx().quantize(_block(-0.0), MX.FLOOR)[0][0, 0] == 8
    assert mx().quantize(_block(2.0 ** -149), MX.CEIL)[1][0, 0] == 0
    big = float(np.finfo(np.float32).max)
    for mode in (MX.FLOOR, MX.CEIL):
        codes, byte = mx().quantize(_block(big, -big), mode)
        assert byte[0, 0] == 252 and codes[0, :2].tolist() == [7, 15]
        assert np.isfinite(mx().values(codes, byte).astype(np.float32)).all()
    for v in (np.inf, -np.inf, np.nan):
        codes, byte = mx().quantize(np.concatenate([_block(v, 1.0), _block(1.0)], axis=1), MX.FLOOR)
        assert byte.tolist() == [[255, 125]] and not codes[0, :32].any()
        got = mx().values(codes, byte)
        assert np.isnan(got[0, :32]).all() and got[0, 32] == 1.0


def pin_every_value_keeps_itself_and_blocks_are_separate():
    rng = np.random.default_rng(5)
    grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    x = grid[rng.integers(0, 8, (7, 70))] * rng.choice([-1, 1], (7, 70)) * np.repeat(2.0 ** rng.integers(-20, 20, (7, 3)), 32, axis=1)[:, :70]
    for mode in (MX.FLOOR, MX.CEIL):
        assert np.array_equal(mx().values(*mx().quantize(x, mode)), x)
        u = rng.integers(0, 256, x.shape)
        assert np.array_equal(mx().values(*mx().quantize(x, mode, u)), x)


def pin_error_bound():
    """Half a step at most: 2^-2 of the value for normal elements, X / 4 below; the scale rules by their definitions."""
    rng = np.random.default_rng(6)
    x = rng.standard_normal((50, 96))
    for mode in (MX.FLOOR, MX.CEIL):
        codes, byte = mx().quantize(x, mode)
        unit = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
        amax = np.abs(x).reshape(50, 3, 32).max(2)
        if mode == MX.FLOOR:
            assert np.array_equal(byte.astype(int) - 127, np.floor(np.log2(amax)).astype(int) - 2)
        else:
            assert (amax <= 6 * 2.0 ** (byte.astype(float) - 127)).all() and (amax > 3 * 2.0 ** (byte.astype(float) - 127)).all()
        err = np.abs(mx().values(codes, byte) - x)
        kept = np.abs(x) <= 6 * unit
        step = np.where(np.abs(x) < 2 * unit, 0.5, np.where(np.abs(x) < 4 * unit, 1.0, 2.0)) * unit
        assert (err[kept] <= step[kept] / 2).all()
        assert np.array_equal(mx().values(codes, byte)[~kept], (np.sign(x) * 6 * unit)[~kept])


def pin_noise_by_its_formula_and_its_mean():
    rng = np.random.default_rng(7)
    a = np.concatenate([rng.uniform(0, 6, 31), [6.0]])
    got = np.zeros((256, 32))
    for u in range(256):
        codes, byte = mx().quantize(a[None], MX.CEIL, np.full((1, 32), u))
        got[u] = mx().values(codes, byte)
        for j, v in enumerate(a):
            s = 0.5 if v < 2 else 1.0 if v < 4 else 2.0
            t = 256 * v / s
            r = math.floor(t)
            r += 1 if t - r > 0.5 or (t - r == 0.5 and r % 2) else 0
            assert got[u, j] == min(6.0, s * ((r + u) // 256))
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert (np.abs(got.mean(0) - a) <= step / 512 + 1e-12).all()


def pin_layout():
    rng = np.random.default_rng(8)
    for rows, cols in ((1, 1), (64, 128), (65, 129), (200, 300)):
        codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
        scales = rng.integers(1, 254, (rows, -(-cols // 32))).astype(np.uint8)
        img = mx().pack(codes, scales)
        assert img.size == mx().image_bytes(rows, cols)
        c, s, clean = mx().unpack(img, rows, cols)
        assert clean and np.array_equal(c, codes) and np.array_equal(s, scales)
    codes = np.zeros((70, 300), dtype=np.uint8)
    codes[67, 128 + 32 * 2 + 5] = 9
    scales = np.zeros((70, 10), dtype=np.uint8)
    scales[67, 6] = 77
    img = mx().pack(codes, scales)
    ks = 3
    # row 67 = 64 + 3: slot 3 of the first unit of the third 32 rows
    assert img[(4 * ks + 1) * 1024 + (2 * 16 + 3) * 16 + 5 // 2] == 9 << 4
    assert img[128 * 384 // 2 + (1 * ks + 1) * 256 + (2 * 16 + 3) * 4 + 0] == 77
    assert np.count_nonzero(img) == 2
    codes[:], scales[:] = 0, 0
    codes[46, 0], scales[46, 0] = 3, 55             # row 46 = 32 + 8 + 4 + 2: slot 4 + 2 of the second unit of the second 32 rows
    other = mx().pack(codes, scales)
    assert other[3 * ks * 1024 + 6 * 16] == 3 and other[128 * 384 // 2 + 6 * 4 + 3] == 55 and np.count_nonzero(other) == 2
    img[3] = 1      # row 0, k 6: not the padding
    assert mx().unpack(img, 70, 300)[2]
    for row64, block, slot, unit in ((1, 0, 15, 3), (0, 11, 0, 0)):      # scales of row 127 and of a padding block
        bad = img.copy()
        bad[128 * 384 // 2 + (row64 * ks + block // 4) * 256 + (block % 4 * 16 + slot) * 4 + unit] = 1
        assert not mx().unpack(bad, 70, 300)[2]


def pin_product():
    a, b, c = np.array([[1.0, 2.0], [3.0, -4.0]]), np.array([[0.5, 1.0]]), np.array([[10.0], [np.nan]])
    assert mx().product(a, b).tolist() == [[2.5], [-2.5]]
    got = mx().product(a, b, 2.0, 0.5, np.array([[10.0], [20.0]]))
    assert got.tolist() == [[10.0], [5.0]]
    assert mx().product(a, b, 2.0, 0.0, c).tolist() == [[5.0], [-5.0]]     # C is not read


PINS = [v for k, v in sorted(globals().items()) if k.startswith("pin_")]


@pytest.mark.parametrize("pin", PINS, ids=lambda f: f.__name__[4:])
def test_pin(pin):
    pin()


MUTANTS = [
    ("amax >= 4.0 * x", "amax > 4.0 * x"),
    ("amax > 6.0 * (x / 2)", "amax >= 6.0 * (x / 2)"),
    ("amax > 6.0 * (x / 2)", "amax > 6.0 * x"),
    ("MIN_EXP, MAX_EXP = -127, 125", "MIN_EXP, MAX_EXP = -126, 125"),
    ("MIN_EXP, MAX_EXP = -127, 125", "MIN_EXP, MAX_EXP = -127, 126"),
    ("np.arange(8) % 2 == 0", "np.arange(8) % 2 == 1"),
    ("np.where(tied.sum(-1) == 2, even.argmax(-1), tied.argmax(-1))", "tied.argmax(-1)"),
    ("side=\"right\") - 1", "side=\"right\")"),
    ("share + u >= 256", "share + u > 256"),
    ("share + u >= 256", "share + u >= 255"),
    ("* 256)", "* 255)"),
    ("code + 8 * np.signbit(v)", "code + 8 * (v < 0)"),
    ("np.where(bad[..., None], 0.0, v)", "np.nan_to_num(v)"),
    ("np.where(bad, NAN_BYTE, e + 127)", "e + 127"),
    ("np.where(codes & 8, -1.0, 1.0)", "1.0"),
    ("np.exp2(scales.astype(np.float64) - 127)", "np.exp2(scales.astype(np.float64) - 126)"),
    ("np.stack([c & 15, c >> 4], axis=-1)", "np.stack([c >> 4, c & 15], axis=-1)"),
    ("c[:, 0::2] | c[:, 1::2] << 4", "c[:, 1::2] | c[:, 0::2] << 4"),
    ("transpose(0, 5, 3, 6, 4, 1, 2)", "transpose(0, 5, 3, 4, 6, 1, 2)"),
    ("not s[rows:].any()", "True"),
    ("return r if beta == 0.0 else r + beta * c", "return r + beta * c if c is not None else r"),
    ("alpha * (a @ b.T)", "a @ b.T"),
]


@pytest.mark.parametrize("old,new", MUTANTS)
def test_planted_mistake_is_caught(old, new):
    src = inspect.getsource(MX)
    assert src.count(old) == 1
    m = types.ModuleType("oracle.mx_mutant")
    m.__package__ = "oracle"
    exec(compile(src.replace(old, new), MX.__file__, "exec"), m.__dict__)
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
        MODULE[0] = MX
    assert caught
