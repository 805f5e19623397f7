"""Host side of the calls around a linear layer (canz_mx_eight_*, canz_act_*, canz_norm_*): sizes, struct layouts, and everything that is refused before any device
work.  CPU only: the calls below never reach a launch."""
import ctypes
import os
import re

import pytest

from oracle import layer as L

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "canz.h")


def _code(canz, fn, *args):
    with pytest.raises(canz.CanzError) as e:
        fn(*args)
    return e.value.code


def test_image_bytes(canz):
    for rows in (0, 1, 63, 1000, 25600):
        for cols in (0, 1, 31, 128, 129, 5120):
            want = L.image_bytes(rows, cols)
            assert canz.canz_mx_eight_bytes(rows, cols) == want and want % 256 == 0
    assert canz.canz_mx_eight_bytes(4194240, 4194240) == L.image_bytes(4194240, 4194240)   # past 32 bits
    assert _code(canz, canz.canz_mx_eight_bytes, -1, 5) == canz.EINVAL
    assert _code(canz, canz.canz_mx_eight_bytes, 5, 4194241) == canz.ESHAPE


def _struct_fields(name):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    sizes = {"int64_t": 8, "int32_t": 4, "float": 4}
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
    fields = []
    for decl in body.split(";"):
        decl = decl.strip()
        if decl:
            kind, names = re.match(r"((?:const )?\w+(?:[\s*]|const)*?)\s*([\w, ]+)$", decl).groups()
            fields += [(n.strip(), 8 if "*" in kind else sizes[kind.strip()]) for n in names.split(",")]
    return fields


@pytest.mark.parametrize("name,struct", [("canz_mx8_group", "_Mx8Group"), ("canz_act", "_Act"), ("canz_act_grad", "_ActGrad"), ("canz_norm", "_Norm"),
                                         ("canz_norm_grad", "_NormGrad")])
def test_struct_layouts_match_header(canz, name, struct):
    struct = getattr(canz, struct)
    assert [(f, ctypes.sizeof(t)) for f, t in struct._fields_] == _struct_fields(name)


def test_images_refusals(canz):
    ok = dict(rows=64, cols=100, mat=[4096], image=[8192])
    for fn in (canz.canz_mx_eight_store, canz.canz_mx_eight_load):
        def f(**kw):
            return _code(canz, fn, [canz.Mx8Group(**{**ok, **kw})], 0)
        assert f(mat=[4097]) == canz.EINVAL
        assert f(mat=[4098], dtype=canz.DT_F32) == canz.EINVAL
        assert f(mat=[0]) == canz.EINVAL
        assert f(image=[8192 + 128]) == canz.EINVAL
        assert f(image=[0]) == canz.EINVAL
        assert f(image=[]) == canz.EINVAL
        assert f(mat=[], image=[], n_mats=1) == canz.EINVAL
        assert f(ld=99) == canz.EINVAL
        assert f(rows=-1) == canz.EINVAL
        assert f(n_mats=-2, mat=[], image=[]) == canz.EINVAL
        assert f(rows=4194241) == canz.ESHAPE
        assert f(rows=4194240, cols=4194240) == canz.ESHAPE
        assert f(rows=131073, cols=131072) == canz.ESHAPE and "2^34" in canz.canz_last_error()
        assert f(rows=131072, cols=131072, mat=[0]) == canz.EINVAL
        assert f(dtype=canz.DT_MX) == canz.EUNSUPPORTED
        assert f(dtype=canz.DT_MX8) == canz.EUNSUPPORTED
        # a later group that is wrong stops the call before the first is enqueued (no device here: a launch would fail otherwise)
        assert _code(canz, fn, [canz.Mx8Group(**ok), canz.Mx8Group(**{**ok, "ld": 1})], 0) == canz.EINVAL
        with pytest.raises(ValueError):
            fn([canz.Mx8Group(rows=64, cols=128, mat=[4096, 8192], image=[16384])], 0)
        fn([], 0)
        fn([canz.Mx8Group(rows=0, cols=5, n_mats=3), canz.Mx8Group(rows=5, cols=0, n_mats=3), canz.Mx8Group(rows=5, cols=5)], 0)


def test_act_refusals(canz):
    ok = dict(rows=64, cols=100, gate=4096, up=8192, out=12288, gate8=16384, up8=20480)

    def f(**kw):
        return _code(canz, canz.canz_act_forward, [canz.Act(**{**ok, **kw})], 0)

    assert f(gate=None) == canz.EINVAL
    assert f(gate=4097) == canz.EINVAL
    assert f(up=8193) == canz.EINVAL
    assert f(out=12290, dtype=canz.DT_F32) == canz.EINVAL
    assert f(gate8=16384 + 64) == canz.EINVAL
    assert f(up8=20480 + 16) == canz.EINVAL
    assert f(up=None) == canz.EINVAL and "up8 without up" in canz.canz_last_error()
    assert f(out=None, gate8=None, up8=None) == canz.EINVAL
    assert f(ld_in=99) == canz.EINVAL
    assert f(ld_out=99) == canz.EINVAL
    assert f(cols=-1) == canz.EINVAL
    assert f(cols=4194241) == canz.ESHAPE
    assert f(act=4) == canz.EUNSUPPORTED
    assert f(act=-1) == canz.EUNSUPPORTED
    assert f(dtype=canz.DT_MX8) == canz.EUNSUPPORTED
    canz.canz_act_forward([], 0)
    canz.canz_act_forward([canz.Act(rows=0, cols=7), canz.Act(rows=7, cols=0)], 0)

    ok2 = dict(rows=64, cols=100, dout=4096, gate=8192, up=12288, dgate=16384, dup=20480, out=24576)

    def b(**kw):
        return _code(canz, canz.canz_act_backward, [canz.ActGrad(**{**ok2, **kw})], 0)

    assert b(gate=8192 + 16) == canz.EINVAL
    assert b(gate=8192 + 2, in_dtype=canz.DT_F32) == canz.EINVAL
    assert b(up=12288 + 64) == canz.EINVAL
    assert b(gate=None) == canz.EINVAL
    assert b(dout=None) == canz.EINVAL
    assert b(dgate=16385) == canz.EINVAL
    assert b(dup=20481) == canz.EINVAL
    assert b(out=24577) == canz.EINVAL
    assert b(dout=4097) == canz.EINVAL
    assert b(up=None) == canz.EINVAL and "dup without up" in canz.canz_last_error()
    assert b(dgate=None, dup=None, out=None) == canz.EINVAL
    assert b(ld_in=99) == canz.EINVAL
    assert b(ld_out=5) == canz.EINVAL
    assert b(rows=4194240, cols=4194240) == canz.ESHAPE
    assert b(in_dtype=canz.DT_MX) == canz.EUNSUPPORTED
    assert b(dtype=canz.DT_MX8) == canz.EUNSUPPORTED
    assert b(act=9) == canz.EUNSUPPORTED
    assert b(dgate=8192) == canz.EINVAL and "another type" in canz.canz_last_error()       # over an image
    assert b(dup=12288, in_dtype=canz.DT_F32) == canz.EINVAL
    canz.canz_act_backward([], 0)
    canz.canz_act_backward([canz.ActGrad(rows=0, cols=7), canz.ActGrad(rows=7, cols=0)], 0)


def test_norm_refusals(canz):
    ok = dict(rows=64, cols=100, x=4096, residual=8192, weight=12288, sum=16384, y=20480, y8=24576, rstd=28672)

    def f(**kw):
        return _code(canz, canz.canz_norm_forward, [canz.Norm(**{**ok, **kw})], 0)

    assert f(x=None) == canz.EINVAL
    assert f(weight=None) == canz.EINVAL
    assert f(weight=None, y=None) == canz.EINVAL
    assert f(x=4097) == canz.EINVAL
    assert f(residual=8193) == canz.EINVAL
    assert f(sum=16384 + 2, sum_dtype=canz.DT_F32) == canz.EINVAL
    assert f(y=20481) == canz.EINVAL
    assert f(weight=12290) == canz.EINVAL
    assert f(y8=24576 + 128) == canz.EINVAL
    assert f(rstd=28674) == canz.EINVAL
    assert f(sum=None, y=None, y8=None, rstd=None) == canz.EINVAL
    assert f(eps=-1.0) == canz.EINVAL
    assert f(eps=float("nan")) == canz.EINVAL
    for ld in ("ldx", "lds", "ldy"):
        assert f(**{ld: 99}) == canz.EINVAL
    assert f(rows=-1) == canz.EINVAL
    assert f(cols=4194241) == canz.ESHAPE
    for t in ("dtype", "sum_dtype", "weight_dtype"):
        assert f(**{t: canz.DT_MX8}) == canz.EUNSUPPORTED
    canz.canz_norm_forward([], 0)
    canz.canz_norm_forward([canz.Norm(rows=0, cols=7), canz.Norm(rows=7, cols=0)], 0)

    ok2 = dict(rows=64, cols=100, dy=4096, h=8192, rstd=12288, weight=16384, dx=20480, dsum=24576, dweight=28672)

    def b(ws=1 << 20, ws_bytes=1 << 40, **kw):
        return _code(canz, canz.canz_norm_backward, [canz.NormGrad(**{**ok2, **kw})], ws, ws_bytes, 0)

    for name in ("dy", "h", "rstd", "weight"):
        assert b(**{name: None}) == canz.EINVAL
    for name in ("dy", "h", "rstd", "weight", "dx", "dsum", "dweight"):
        assert b(**{name: ok2[name] + 1}) == canz.EINVAL
    assert b(h=8192 + 128, h_dtype=canz.DT_MX8) == canz.EINVAL
    assert b(dx=None, dweight=None) == canz.EINVAL
    assert b(ldy=99) == canz.EINVAL
    assert b(lds=99) == canz.EINVAL
    assert b(rows=4194241) == canz.ESHAPE
    assert b(h_dtype=canz.DT_MX) == canz.EUNSUPPORTED
    for t in ("dtype", "sum_dtype", "weight_dtype"):
        assert b(**{t: canz.DT_MX8}) == canz.EUNSUPPORTED
    assert b(ws=0) == canz.EWORKSPACE
    assert b(ws=(1 << 20) + 128) == canz.EWORKSPACE
    need = canz.canz_norm_backward_workspace_bytes([canz.NormGrad(**ok2)])
    assert need >= 256 and b(ws_bytes=need - 1) == canz.EWORKSPACE
    assert canz.canz_norm_backward_workspace_bytes([]) == 256
    assert canz.canz_norm_backward_workspace_bytes([canz.NormGrad(**{**ok2, "dweight": None, "rows": 4096, "cols": 4096})]) == 256
    assert _code(canz, canz.canz_norm_backward_workspace_bytes, [canz.NormGrad(rows=-1, cols=5)]) == canz.EINVAL
    canz.canz_norm_backward([], 0, 0, 0)
    canz.canz_norm_backward([canz.NormGrad(rows=5, cols=0)], 0, 0, 0)
    assert b(rows=0, dx=None, dweight=None) == canz.EINVAL
    assert b(rows=0, ws=0) == canz.EWORKSPACE          # dweight <- beta dweight is left to do


def test_linear_struct_layout(canz):
    assert [(f, ctypes.sizeof(t)) for f, t in canz._Linear._fields_] == _struct_fields("canz_linear_group")


def test_linear_refusals_and_workspace(canz):
    P = canz.Linear
    ok = dict(m=80, n=128, k=256, a=[4096], b=[8192], c=[12288])

    def p(ws=256 * 1024, ws_bytes=1 << 40, **kw):
        return _code(canz, canz.canz_linear, [P(**{**ok, **kw})], ws, ws_bytes, 0)

    assert p(a=[4097]) == canz.EINVAL
    assert p(b=[8193]) == canz.EINVAL
    assert p(a=[4096 + 64], a_dtype=canz.DT_MX8) == canz.EINVAL
    assert p(b=[8192 + 128], b_dtype=canz.DT_MX8) == canz.EINVAL
    assert p(a=[0]) == canz.EINVAL
    assert p(c=[0]) == canz.EINVAL
    assert p(c=[12290], out_dtype=canz.DT_F32) == canz.EINVAL
    assert p(bias=[0]) == canz.EINVAL
    assert p(bias=[4098]) == canz.EINVAL
    assert p(residual=[0]) == canz.EINVAL
    assert p(residual=[4097]) == canz.EINVAL
    assert p(residual=[16384], ldr=127) == canz.EINVAL
    assert p(residual=[12288], ldr=129) == canz.EINVAL and "another row distance" in canz.canz_last_error()
    assert p(pre8=[16384 + 16]) == canz.EINVAL
    assert p(a_sums=[16386]) == canz.EINVAL
    assert p(a_sums=[0]) == canz.EINVAL
    assert p(a=[], n_prods=1) == canz.EINVAL
    assert p(m=-1) == canz.EINVAL
    assert p(ldc=127) == canz.EINVAL
    assert p(lda=255) == canz.EINVAL
    assert p(lda=79, a_trans=True) == canz.EINVAL
    assert p(ldb=127, b_trans=True) == canz.EINVAL
    assert p(a_trans=2) == canz.EINVAL
    assert p(b_trans=-1) == canz.EINVAL
    assert p(n_prods=-2, a=[], b=[], c=[]) == canz.EINVAL
    assert p(n=4194241) == canz.ESHAPE
    assert p(n=4194240, k=4194240) == canz.ESHAPE
    assert p(a_dtype=canz.DT_F32) == canz.EUNSUPPORTED
    assert p(b_dtype=canz.DT_MX) == canz.EUNSUPPORTED
    assert p(out_dtype=canz.DT_MX8) == canz.EUNSUPPORTED
    assert p(bias_dtype=canz.DT_MX8) == canz.EUNSUPPORTED
    assert p(act=4) == canz.EUNSUPPORTED
    assert p(ws=0) == canz.EWORKSPACE
    assert p(ws=256 + 16) == canz.EWORKSPACE
    assert p(ws_bytes=255) == canz.EWORKSPACE
    # operands that lie well need nothing, others a copy of their own, and so do tables that are not given
    w = canz.canz_linear_workspace_bytes
    base = w([P(**ok)])
    assert base >= 256
    assert w([P(**{**ok, "a": [4098]})]) >= base + 80 * 256 * 2 - 256
    assert w([P(**{**ok, "ldb": 257})]) >= base + 128 * 256 * 2 - 256
    assert w([P(m=80, n=128, k=256, n_prods=1)]) >= base + (80 + 128) * 256 * 2 - 512
    assert w([P(m=64, n=128, k=257, n_prods=1)]) == 256                       # few rows are read where they lie
    assert w([P(m=64, n=128, k=257, n_prods=3, b_dtype=canz.DT_MX8)]) >= 3 * 128 * 257 * 2
    assert p(a=[4098], ws_bytes=w([P(**{**ok, "a": [4098]})]) - 1) == canz.EWORKSPACE
    assert "workspace too small" in canz.canz_last_error()
    assert w([]) == 256
    assert _code(canz, w, [P(m=1, n=1, k=-1, n_prods=1)]) == canz.EINVAL
    many = dict(m=1 << 17, n=128, k=1 << 17, n_prods=(1 << 31) - 1)
    assert _code(canz, w, [P(**many)]) == canz.ESHAPE and "64 bits" in canz.canz_last_error()
    for extents in (dict(m=131073, n=131072, k=1), dict(m=131073, n=1, k=131072), dict(m=1, n=131073, k=131072)):
        assert _code(canz, w, [P(n_prods=1, **extents)]) == canz.ESHAPE and "2^34" in canz.canz_last_error()
    assert w([P(m=131072, n=131072, k=0, n_prods=1)]) == 256
    # a later group that is wrong stops the call before the first is enqueued (no device here: a launch would fail otherwise)
    assert _code(canz, canz.canz_linear, [P(**ok), P(**{**ok, "ldc": 1})], 256 * 1024, 1 << 40, 0) == canz.EINVAL
    with pytest.raises(ValueError):
        canz.canz_linear([P(**{**ok, "bias": [4096, 4096]})], 256 * 1024, 1 << 40, 0)
    # nothing to do: neither pointers nor a workspace are looked at
    canz.canz_linear([], 0, 0, 0)
    canz.canz_linear([P(m=0, n=5, k=5, n_prods=2), P(m=5, n=0, k=5, n_prods=2), P(m=5, n=5, k=5, n_prods=0)], 0, 0, 0)
