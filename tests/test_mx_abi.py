"""Host side of canz_mx_* and canz_muon_step_images: sizes, struct layouts, and everything that is refused before any device work.
CPU only: the calls below never reach a launch."""
import ctypes
import os
import re

import pytest

from oracle import mx as MX

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "canz.h")


def _code(canz, fn, *args):
    with pytest.raises(canz.CanzError) as e:
        fn(*args)
    return e.value.code


def test_image_bytes(canz):
    for rows in (0, 1, 63, 64, 65, 1000, 25600):
        for cols in (0, 1, 31, 32, 127, 128, 129, 5120):
            want = MX.image_bytes(rows, cols)
            assert canz.canz_mx_image_bytes(rows, cols) == want and want % 256 == 0
    assert canz.canz_mx_image_bytes(4194240, 4194240) == MX.image_bytes(4194240, 4194240)   # past 32 bits
    assert _code(canz, canz.canz_mx_image_bytes, -1, 5) == canz.EINVAL
    assert _code(canz, canz.canz_mx_image_bytes, 5, 4194241) == canz.ESHAPE


def test_struct_layouts_match_header(canz):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    sizes = {"int64_t": 8, "int32_t": 4, "float": 4}
    for name, struct in (("canz_mx_group", canz._MxGroup), ("canz_mx_product_group", canz._MxProduct), ("canz_mx_images", canz._MxImages)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
        fields = []
        for decl in body.split(";"):
            decl = decl.strip()
            if decl:
                kind, names = re.match(r"((?:const )?\w+(?:[\s*]|const)*?)\s*([\w, ]+)$", decl).groups()
                fields += [(n.strip(), 8 if "*" in kind else sizes[kind.strip()]) for n in names.split(",")]
        assert [f for f, _ in fields] == [f for f, _ in struct._fields_]
        assert [s for _, s in fields] == [ctypes.sizeof(t) for _, t in struct._fields_]
        assert sum(s for _, s in fields) == ctypes.sizeof(struct)


def test_quantize_and_dequantize_refusals(canz):
    G = canz.MxGroup
    ok = dict(rows=64, cols=128, mat=[4096], by_row=[8192])

    def q(mode=0, **kw):
        return _code(canz, canz.canz_mx_quantize, [G(**{**ok, **kw})], mode, 0)

    def d(**kw):
        return _code(canz, canz.canz_mx_dequantize, [G(**{**ok, **kw})], 0)

    for f in (q, d):
        assert f(mat=[4100]) == canz.EINVAL
        assert f(mat=[0]) == canz.EINVAL
        assert f(by_row=[8192 + 16]) == canz.EINVAL
        assert f(by_row=[0]) == canz.EINVAL
        assert f(by_row=[], by_col=[8200]) == canz.EINVAL
        assert f(by_row=[]) == canz.EINVAL
        assert f(mat=[], n_mats=1) == canz.EINVAL
        assert f(ld=127) == canz.EINVAL
        assert f(rows=-1) == canz.EINVAL
        assert f(n_mats=-2, mat=[], by_row=[]) == canz.EINVAL
        assert f(rows=4194241) == canz.ESHAPE
        assert f(rows=4194240, cols=4194240) == canz.ESHAPE
        assert f(dtype=canz.DT_MX) == canz.EUNSUPPORTED
        assert f(dtype=-1) == canz.EUNSUPPORTED
    assert q(mode=2) == canz.EUNSUPPORTED
    assert q(mode=-1) == canz.EUNSUPPORTED
    assert q(noise=[0]) == canz.EINVAL
    assert d(by_col=[16384]) == canz.EINVAL
    assert "both are given" in canz.canz_last_error()
    # a later group that is wrong stops the call before the first is enqueued (no device here: a launch would fail otherwise)
    assert _code(canz, canz.canz_mx_quantize, [G(**ok), G(**{**ok, "ld": 1})], 0, 0) == canz.EINVAL
    with pytest.raises(ValueError):
        canz.canz_mx_quantize([G(rows=64, cols=128, mat=[4096, 8192], by_row=[16384])], 0, 0)
    # nothing to do: no pointer is looked at
    canz.canz_mx_quantize([], 0, 0)
    canz.canz_mx_dequantize([], 0)
    for kw in (dict(rows=0, cols=5), dict(rows=5, cols=0)):
        canz.canz_mx_quantize([G(n_mats=3, **kw)], 0, 0)
        canz.canz_mx_dequantize([G(n_mats=3, **kw)], 0)


def test_product_refusals_and_workspace(canz):
    P = canz.MxProduct
    ok = dict(m=64, n=128, k=256, a=[4096], b=[8192], c=[12288])

    def p(ws=256 * 1024, ws_bytes=1 << 40, **kw):
        return _code(canz, canz.canz_mx_product, [P(**{**ok, **kw})], ws, ws_bytes, 0)

    assert p(a=[4096 + 16]) == canz.EINVAL                                    # an image
    assert p(a=[4096 + 8], a_dtype=canz.DT_BF16) == canz.EINVAL
    assert p(b=[8192 + 16]) == canz.EINVAL
    assert p(b=[0]) == canz.EINVAL
    assert p(c=[12292]) == canz.EINVAL
    assert p(a=[], n_prods=1) == canz.EINVAL
    assert p(m=-1) == canz.EINVAL
    assert p(ldc=127) == canz.EINVAL
    assert p(lda=255, a_dtype=canz.DT_F32) == canz.EINVAL
    assert p(n_prods=-2, a=[], b=[], c=[]) == canz.EINVAL
    assert p(n=4194241) == canz.ESHAPE
    assert p(n=4194240, k=4194240) == canz.ESHAPE
    assert p(a_dtype=3) == canz.EUNSUPPORTED
    assert p(out_dtype=canz.DT_MX) == canz.EUNSUPPORTED
    assert p(a_scale_mode=2) == canz.EUNSUPPORTED
    assert p(ws=0) == canz.EWORKSPACE
    assert p(ws=256 + 16) == canz.EWORKSPACE
    assert p(ws_bytes=255) == canz.EWORKSPACE
    need = canz.canz_mx_product_workspace_bytes([P(m=640, n=128, k=256, n_prods=3, a_dtype=canz.DT_BF16)])
    assert need >= 3 * canz.canz_mx_image_bytes(640, 256)
    assert p(a_dtype=canz.DT_BF16, ws_bytes=canz.canz_mx_product_workspace_bytes([P(m=64, n=128, k=256, n_prods=1, a_dtype=canz.DT_BF16)]) - 1) \
        == canz.EWORKSPACE
    assert "workspace too small" in canz.canz_last_error()
    assert canz.canz_mx_product_workspace_bytes([]) >= 256
    assert _code(canz, canz.canz_mx_product_workspace_bytes, [P(m=1, n=1, k=-1, n_prods=1)]) == canz.EINVAL
    # nothing to do: neither pointers nor a workspace are looked at
    canz.canz_mx_product([], 0, 0, 0)
    canz.canz_mx_product([P(m=0, n=5, k=5, n_prods=2), P(m=5, n=0, k=5, n_prods=2), P(m=5, n=5, k=5, n_prods=0)], 0, 0, 0)


def test_workspace_past_64_bits_is_refused(canz):
    P = canz.MxProduct
    many = dict(m=1 << 18, n=128, k=1 << 19, n_prods=(1 << 31) - 1, a_dtype=canz.DT_BF16)   # 7.3e10 bytes of image each
    assert canz.canz_mx_product_workspace_bytes([P(**{**many, "n_prods": 1000})]) >= 1000 * canz.canz_mx_image_bytes(1 << 18, 1 << 19)
    assert _code(canz, canz.canz_mx_product_workspace_bytes, [P(**many)]) == canz.ESHAPE
    assert _code(canz, canz.canz_mx_product_workspace_bytes, [P(**{**many, "n_prods": 1 << 27})] * 3) == canz.ESHAPE   # their sum


def test_tables_may_be_any_sequence(canz):
    np = pytest.importorskip("numpy")
    for kind in (tuple, np.array):
        assert _code(canz, canz.canz_mx_quantize, [canz.MxGroup(rows=64, cols=128, mat=kind([4096, 8192]), by_row=kind([8192, 8200]))], 0, 0) == canz.EINVAL
        assert "by_row[1]" in canz.canz_last_error()


def test_step_images_refusals(canz):
    ok = dict(rows=256, cols=512, grad=[4096], mom=[8192], out=[12288])

    def s(img, hp=None, mode=0, ws=256 * 1024, ws_bytes=1 << 40, **kw):
        return _code(canz, canz.canz_muon_step_images, [canz.Group(**{**ok, **kw})], hp or canz.Hparams(), [img], mode, ws, ws_bytes, 0)

    good = canz.MxImages(by_row=[16384])
    assert s(good, hp=canz.Hparams(out_mode=canz.OUT_DELTA)) == canz.EUNSUPPORTED
    assert s(good, mode=5) == canz.EUNSUPPORTED
    assert s(canz.MxImages(by_row=[16384 + 16])) == canz.EINVAL
    assert s(canz.MxImages(by_col=[0])) == canz.EINVAL
    assert s(good, grad=[4100]) == canz.EINVAL                                # the step's own checks
    assert s(good, hp=canz.Hparams(ns_steps=-1)) == canz.EINVAL
    assert s(good, ws=0) == canz.EWORKSPACE
    assert s(good, out_dtype=7) == canz.EUNSUPPORTED
    assert s(good, rows=0) == canz.EINVAL
    with pytest.raises(ValueError):
        canz.canz_muon_step_images([canz.Group(**ok)], canz.Hparams(), [], 0, 256 * 1024, 1 << 40, 0)
    canz.canz_muon_step_images([], canz.Hparams(), [], 0, 0, 0, 0)
