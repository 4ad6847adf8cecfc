"""Root-mean-square norm, rows in 8 bits and their products without a GPU: layout of the descriptors, what is refused, what workspaces are asked for, and that no refused call
launches anything."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2006_06762_amd import binding as B  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, P2, P3, ODD = (ctypes.c_void_p(v) for v in (0x10000, 0x20000, 0x30000, 0x10001))      # never dereferenced: validation fails first
OK, NULL, INVALID, UNSUPPORTED, WORKSPACE = B.ANR_OK, B.ANR_ERR_NULL, B.ANR_ERR_INVALID_ARG, B.ANR_ERR_UNSUPPORTED, B.ANR_ERR_WORKSPACE


def layout_of(tmp_path, fields):
    """(sizes and offsets as C has them, as the binding has them)."""
    text = '#include <stdio.h>\n#include <stddef.h>\n#include "anr.h"\nint main(void) {\n'
    want = []
    for c, t in fields.items():
        text += 'printf("%%zu ", sizeof(%s));\n' % c
        want.append(ctypes.sizeof(t))
        for n, *_ in t._fields_:
            text += 'printf("%%zu ", offsetof(%s, %s));\n' % (c, n)
            want.append(getattr(t, n).offset)
    (tmp_path / "l.c").write_text(text + "return 0; }")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    return [int(v) for v in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.split()], want


def test_layouts_match_c(tmp_path):
    got, want = layout_of(tmp_path, {"anr_rms_norm_desc": B.RmsNormDesc, "anr_rows_q8_desc": B.RowsQ8Desc, "anr_gemm_i8_desc": B.GemmI8Desc})
    assert got == want


def norm_desc(**kw):
    return B.RmsNormDesc(**dict(dict(T=9, C=40, dtype=B.ANR_BF16, param_dtype=B.ANR_BF16), **kw))


def norm(d, x=P, residual=None, gamma=P, eps=1e-6, h=None, y=P2, rstd=None):
    return B.raw().anr_rms_norm(ctypes.byref(d) if d else None, x, residual, gamma, ctypes.c_float(eps), h, y, rstd, None, 0, None)


def norm_q8(d, x=P, residual=None, gamma=P, eps=1e-6, h=None, y=P2, scale=P3):
    return B.raw().anr_rms_norm_q8(ctypes.byref(d) if d else None, x, residual, gamma, ctypes.c_float(eps), h, y, scale, None, 0, None)


def norm_backward(d, dy=P, x=P2, gamma=P, rstd=P, dh=None, dx=P3, dgamma=P, ws=None, size=0):
    return B.raw().anr_rms_norm_backward(ctypes.byref(d) if d else None, dy, x, gamma, rstd, dh, dx, dgamma, ws, size, None)


def test_rms_norm_refusals():
    for call in (norm, norm_q8, norm_backward):
        assert call(None) == NULL
        for field, bad in (("T", -1), ("C", 0), ("dtype", 3), ("dtype", -1), ("param_dtype", B.ANR_F16), ("ldx", 39), ("ldx", -40), ("ld_residual", 1), ("ldh", 39), ("ldy", 39)):
            assert call(norm_desc(**{field: bad})) == INVALID, (call, field, bad)
        for field, bad in (("C", 32769), ("T", 1 << 31), ("ldx", 1 << 40), ("ldy", 1 << 55)):
            assert call(norm_desc(**{field: bad})) == UNSUPPORTED, (call, field, bad)
        assert call(norm_desc(), x=None) == NULL and call(norm_desc(), x=ODD) == INVALID and call(norm_desc(), gamma=ODD) == INVALID
    for call in (norm, norm_q8):
        assert call(norm_desc(), y=None) == NULL
        for eps in (-1e-9, float("nan"), float("inf")):
            assert call(norm_desc(), eps=eps) == INVALID
        assert call(norm_desc(), h=P3) == INVALID                                    # a sum without a residual
        assert call(norm_desc(), residual=P3, h=ODD) == INVALID and call(norm_desc(), residual=ODD) == INVALID
        assert call(norm_desc(), residual=P3, h=P2) == INVALID                       # two outputs in one place
        assert call(norm_desc(ldx=48), residual=P3, h=P) == INVALID                  # in place with another leading dimension
        assert call(norm_desc(ld_residual=48), residual=P3, h=P3) == INVALID
    assert norm(norm_desc(), y=ODD) == INVALID and norm(norm_desc(), rstd=ctypes.c_void_p(0x10002)) == INVALID
    assert norm(norm_desc(ldy=48), y=P) == INVALID and norm(norm_desc(ldy=48), residual=P2) == INVALID
    assert norm_q8(norm_desc(), scale=None) == NULL and norm_q8(norm_desc(), scale=ctypes.c_void_p(0x10002)) == INVALID
    assert norm_q8(norm_desc(), y=P) == INVALID and norm_q8(norm_desc(), residual=P2) == INVALID
    for name in ("dy", "rstd"):
        assert norm_backward(norm_desc(), **{name: None}) == NULL
    assert norm_backward(norm_desc(), dx=None, dgamma=None) == NULL
    for name in ("dy", "rstd", "dh", "dx", "dgamma"):
        assert norm_backward(norm_desc(), **{name: ODD}) == INVALID, name
    for field, name in (("ldy", "dy"), ("ldx", "x"), ("ld_residual", "dh")):
        assert norm_backward(norm_desc(**{field: 48}), **{name: P3}) == INVALID, field
    d = norm_desc(T=5000)
    need = B.workspace_size(B.ANR_OP_RMS_NORM_BACKWARD, d)
    assert need > 0 and need % 4 == 0
    assert norm_backward(d) == WORKSPACE and norm_backward(d, ws=P, size=need - 1) == WORKSPACE and norm_backward(d, ws=ctypes.c_void_p(0x10008), size=need) == INVALID
    for op in (B.ANR_OP_RMS_NORM, B.ANR_OP_RMS_NORM_Q8):
        assert B.workspace_size(op, d) == 0
    # nothing to do is no error and no launch
    d = norm_desc(T=0)
    assert norm(d, None, y=None) == OK and norm_q8(d, None, y=None, scale=None) == OK and norm_backward(d, None, None, None, None, None, None, None) == OK
    assert B.workspace_size(B.ANR_OP_RMS_NORM_BACKWARD, d) == 0
    # the leading dimensions of a single row say nothing
    assert B.workspace_size(B.ANR_OP_RMS_NORM, norm_desc(T=1, ldx=1, ldy=1 << 60)) == 0


def test_rms_norm_binding_refuses():
    x, g = torch.zeros(4, 8), torch.zeros(8)
    for args, kw, error in (((x, x), {}, TypeError), ((x.double(), x), {}, TypeError), ((x[0], x), {}, ValueError), ((x, x, g.half()), {}, TypeError),
                            ((x, x), {"h": x}, ValueError)):
        with pytest.raises(error):
            B.rms_norm(*args, **kw)
    with pytest.raises(TypeError):
        B.rms_norm_q8(x, x.char(), g[:4])
    with pytest.raises(ValueError):
        B.rms_norm_q8(x, x.char(), g[:4], h=x)
    with pytest.raises(TypeError):
        B.rms_norm_backward(x, x, g, g[:4], x, g.half())


def rows_desc(**kw):
    return B.RowsQ8Desc(**dict(dict(T=9, C=40, act=B.ANR_ACT_NONE, dtype=B.ANR_F16), **kw))


def quantize(d, x=P, up=None, q=P2, scale=P3):
    return B.raw().anr_quantize_rows(ctypes.byref(d) if d else None, x, up, q, scale, None, 0, None)


def dequantize(d, q=P2, scale=P3, x=P):
    return B.raw().anr_dequantize_rows(ctypes.byref(d) if d else None, q, scale, x, None, 0, None)


def test_rows_q8_refusals():
    for call in (quantize, dequantize):
        assert call(None) == NULL
        for field, bad in (("T", -1), ("C", 0), ("act", 5), ("act", -1), ("dtype", 3), ("ldx", 39), ("ldq", -1)):
            assert call(rows_desc(**{field: bad})) == INVALID, (call, field, bad)
        for field, bad in (("C", (1 << 20) + 1), ("T", 1 << 31), ("ldx", 1 << 40), ("ldq", 1 << 60)):
            assert call(rows_desc(**{field: bad})) == UNSUPPORTED, (call, field, bad)
        for name in ("x", "q", "scale"):
            assert call(rows_desc(), **{name: None}) == NULL
        assert call(rows_desc(), x=ODD) == INVALID and call(rows_desc(), scale=ctypes.c_void_p(0x10002)) == INVALID and call(rows_desc(), x=P2) == INVALID
        assert call(rows_desc(T=0), **dict.fromkeys(("x", "q", "scale"))) == OK
    assert quantize(rows_desc(), up=ODD) == INVALID and quantize(rows_desc(), up=P2) == INVALID and quantize(rows_desc(ld_up=39), up=P) == INVALID
    assert dequantize(rows_desc(act=B.ANR_ACT_SILU)) == INVALID
    for op in (B.ANR_OP_QUANTIZE_ROWS, B.ANR_OP_DEQUANTIZE_ROWS):
        assert B.workspace_size(op, rows_desc()) == 0
        with pytest.raises(B.AnrError):
            B.workspace_size(op, rows_desc(ldq=39))


def test_rows_q8_binding_refuses():
    x, s = torch.zeros(4, 8), torch.zeros(4)
    for args in ((x, x.char(), s), (x.char(), x.char(), s), (x, x, s)):
        with pytest.raises(TypeError):
            B.quantize_rows(*args)
    with pytest.raises(ValueError):
        B.quantize_rows(x[0], x.char(), s)
    with pytest.raises(TypeError):
        B.dequantize_rows(x.char(), s, x.double())


def product_desc(**kw):
    return B.GemmI8Desc(**dict(dict(M=9, N=50, K=64, dtype=B.ANR_BF16, bias_dtype=B.ANR_F32), **kw))


def product(d, a=P, w=P2, a_scale=None, w_scale=None, bias=None, out=P3, ws=None, size=0):
    return B.raw().anr_gemm_i8(ctypes.byref(d) if d else None, a, w, a_scale, w_scale, bias, out, ws, size, None)


def test_gemm_i8_refusals():
    assert product(None) == NULL
    for field, bad in (("M", -1), ("N", 0), ("K", 0), ("dtype", 3), ("bias_dtype", B.ANR_F16), ("lda", 63), ("ldw", 63), ("ldd", 49), ("lda", -64)):
        assert product(product_desc(**{field: bad})) == INVALID, (field, bad)
    for field, bad in (("M", 1 << 22), ("N", (1 << 20) + 1), ("K", 1 << 17), ("lda", 1 << 22), ("ldw", 1 << 22), ("ldd", 1 << 22)):
        assert product(product_desc(**{field: bad})) == UNSUPPORTED, (field, bad)
    for name in ("a", "w", "out"):
        assert product(product_desc(), **{name: None}) == NULL
    off = ctypes.c_void_p(0x40002)
    for name in ("a_scale", "w_scale", "bias"):
        assert product(product_desc(), **{name: off}) == INVALID
    assert product(product_desc(), out=ODD) == INVALID
    for name in ("a", "w", "a_scale", "w_scale", "bias"):
        assert product(product_desc(), **{name: P3}) == INVALID              # the result over an input
    assert product(product_desc(M=0), None, None, out=None) == OK
    assert B.workspace_size(B.ANR_OP_GEMM_I8, product_desc(M=0)) == 0 and B.workspace_size(B.ANR_OP_GEMM_I8, product_desc()) == 0
    d = product_desc(M=200, N=300, K=20000)
    need = B.workspace_size(B.ANR_OP_GEMM_I8, d)
    assert need > 0 and need % 4 == 0
    assert product(d) == WORKSPACE and product(d, ws=P, size=need - 1) == WORKSPACE and product(d, ws=ctypes.c_void_p(0x10008), size=need) == INVALID
    # the leading dimensions of a single row say nothing
    assert B.workspace_size(B.ANR_OP_GEMM_I8, product_desc(M=1, lda=1, ldd=1 << 40)) == 0


def test_gemm_i8_binding_refuses():
    a, d, s = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 4), torch.zeros(4)
    for args in ((a, a, s, s, d), (a.float(), a, s, s, d), (a, a, s, s, d.double()), (a, a, s, s, d, s.half()), (a, a, s, s, a)):
        with pytest.raises(TypeError):
            B.gemm_i8(*args)
    with pytest.raises(ValueError):
        B.gemm_i8(a[0], a, s, s, d)
