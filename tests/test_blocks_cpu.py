"""Group norm, rotary positions and the gated feed-forward block without a GPU: layouts of the descriptors, what is refused,
what workspaces are asked for, and that no refused call launches anything."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2006_06762_amd import binding as B  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x10000)            # never dereferenced: validation fails first
OK, NULL, INVALID, UNSUPPORTED, WORKSPACE = B.ANR_OK, B.ANR_ERR_NULL, B.ANR_ERR_INVALID_ARG, B.ANR_ERR_UNSUPPORTED, B.ANR_ERR_WORKSPACE


def test_struct_layouts_match_c(tmp_path):
    fields = {"anr_group_norm_desc": (B.GroupNormDesc, "N groups param_dtype x_stride y_stride dx_stride"),
              "anr_rotary_desc": (B.RotaryDesc, "D axes section pairing inverse pos_type reserved q_stride k_out_stride pos_stride"),
              "anr_gated_ff_desc": (B.GatedFfDesc, "F act dtype ldx ldpre lddx ldw ld_down lddw ld_ddown")}
    text = '#include <stdio.h>\n#include <stddef.h>\n#include "anr.h"\nint main(void) {\n'
    want = []
    for c, (t, names) in fields.items():
        text += 'printf("%%zu ", sizeof(%s));\n' % c
        want.append(ctypes.sizeof(t))
        for n in names.split():
            text += 'printf("%%zu ", offsetof(%s, %s));\n' % (c, n)
            want.append(getattr(t, n).offset)
    (tmp_path / "l.c").write_text(text + "return 0; }")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    assert [int(v) for v in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.split()] == want


def norm_desc(**kw):
    base = dict(N=2, H=4, W=5, C=24, groups=4, act=B.ANR_ACT_SILU, dtype=B.ANR_BF16, param_dtype=B.ANR_BF16)
    strides = {k: kw.pop(k) for k in ("x_stride", "y_stride", "dx_stride") if k in kw}
    d = B.GroupNormDesc(**dict(base, **kw))
    for k, v in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*v))
    return d


def norm(d, x=P, gamma=P, beta=P, eps=1e-5, y=P, mean=P, rstd=P, ws=None, size=0):
    return B.raw().anr_group_norm(ctypes.byref(d) if d else None, x, gamma, beta, ctypes.c_float(eps), y, mean, rstd, ws, size, None)


def norm_backward(d, dy=P, x=P, gamma=P, beta=P, mean=P, rstd=P, dx=P, dgamma=P, dbeta=P, ws=None, size=0):
    return B.raw().anr_group_norm_backward(ctypes.byref(d) if d else None, dy, x, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws, size, None)


def test_group_norm_refusals():
    for call in (norm, norm_backward):
        assert call(None) == NULL
        for field, bad in (("N", -1), ("H", -1), ("W", -2), ("C", 0), ("groups", 0), ("groups", 5), ("act", 5), ("act", -1), ("dtype", 3), ("dtype", -1),
                           ("param_dtype", B.ANR_F16), ("param_dtype", 7)):
            assert call(norm_desc(**{field: bad})) == INVALID, (field, bad)
        assert call(norm_desc(C=16384, groups=1)) == UNSUPPORTED
        assert call(norm_desc(N=70000)) == UNSUPPORTED
        assert call(norm_desc(H=1 << 16, W=1 << 15)) == UNSUPPORTED
        assert call(norm_desc(x_stride=(480, 120, 23))) == INVALID          # pixels overlap
        assert call(norm_desc(x_stride=(480, 119, 24))) == INVALID          # rows overlap
        assert call(norm_desc(x_stride=(479, 120, 24))) == INVALID          # images overlap
        assert call(norm_desc(y_stride=(480, 120, 0))) == INVALID
        assert call(norm_desc(y_stride=(480, -120, 24))) == INVALID
        assert call(norm_desc(x_stride=(1 << 41, 120, 24))) == UNSUPPORTED
        assert call(norm_desc(), x=None) == NULL
        assert call(norm_desc(), x=ctypes.c_void_p(0x10001)) == INVALID
        assert call(norm_desc(), gamma=ctypes.c_void_p(0x10001)) == INVALID
        assert call(norm_desc(), mean=ctypes.c_void_p(0x10002)) == INVALID
        assert call(norm_desc()) == WORKSPACE
    assert norm_backward(norm_desc(dx_stride=(480, 119, 24))) == INVALID
    assert norm(norm_desc(), y=None) == NULL
    assert norm(norm_desc(), eps=-1e-5) == INVALID and norm(norm_desc(), eps=float("nan")) == INVALID and norm(norm_desc(), eps=float("inf")) == INVALID
    assert norm_backward(norm_desc(), dx=None, dgamma=None, dbeta=None) == NULL
    assert norm_backward(norm_desc(), mean=None) == NULL and norm_backward(norm_desc(), rstd=None) == NULL and norm_backward(norm_desc(), dy=None) == NULL
    for call, op in ((norm, B.ANR_OP_GROUP_NORM), (norm_backward, B.ANR_OP_GROUP_NORM_BACKWARD)):
        d = norm_desc(N=4, H=300, W=200)
        need = B.workspace_size(op, d)
        assert need > 0
        assert call(d, ws=P, size=need - 1) == WORKSPACE and call(d, ws=ctypes.c_void_p(0x10008), size=need) == INVALID


def rotary_desc(**kw):
    base = dict(B=2, S=3, H=4, Hk=2, D=32, axes=2, pairing=0, inverse=0, dtype=B.ANR_F16, pos_type=B.ANR_POS_I64, reserved=0)
    arrays = {k: kw.pop(k) for k in ("section", "q_stride", "k_stride", "q_out_stride", "k_out_stride", "pos_stride") if k in kw}
    d = B.RotaryDesc(**dict(base, **kw))
    d.section = (ctypes.c_int32 * 4)(8, 8, 0, 0)
    for k, v in arrays.items():
        setattr(d, k, (ctypes.c_int32 * 4)(*v) if k == "section" else (ctypes.c_int64 * 3)(*v))
    return d


def rotary(d, q=P, k=P, pos=P, freq=P, q_out=ctypes.c_void_p(0x20000), k_out=ctypes.c_void_p(0x30000)):
    return B.raw().anr_rotary(ctypes.byref(d) if d else None, q, k, pos, freq, q_out, k_out, None, 0, None)


def test_rotary_refusals():
    assert rotary(None) == NULL
    for field, bad in (("B", -1), ("S", -1), ("H", -1), ("Hk", -1), ("D", 0), ("D", 31), ("axes", 0), ("axes", 5), ("pairing", 3), ("pairing", -1), ("inverse", 2),
                       ("dtype", 3), ("pos_type", 3), ("pos_type", -1), ("reserved", 1), ("section", (8, -1, 0, 0)), ("section", (9, 8, 0, 0)),
                       ("section", (2147483647, 2147483647, 2, 0)), ("q_stride", (384, 128, -1)), ("pos_stride", (-1, 0, 1)), ("q_out_stride", (384, 128, 31)),
                       ("q_out_stride", (384, 127, 32)), ("k_out_stride", (191, 64, 32)), ("k_out_stride", (0, 64, 32))):
        assert rotary(rotary_desc(**{field: bad})) == INVALID, (field, bad)
    assert rotary(rotary_desc(D=2050)) == UNSUPPORTED
    assert rotary(rotary_desc(B=1 << 16, S=1 << 15)) == UNSUPPORTED
    assert rotary(rotary_desc(H=70000)) == UNSUPPORTED
    assert rotary(rotary_desc(k_stride=(1 << 50, 64, 32))) == UNSUPPORTED
    assert rotary(rotary_desc(pos_stride=(1 << 50, 0, 1))) == UNSUPPORTED
    for name in ("q", "k", "pos", "freq", "q_out", "k_out"):
        assert rotary(rotary_desc(), **{name: None}) == NULL, name
        assert rotary(rotary_desc(), **{name: ctypes.c_void_p(0x10001)}) == INVALID, name
    # in place with other strides
    assert rotary(rotary_desc(q_stride=(512, 160, 32)), q_out=P) == INVALID
    # nothing to do is no error and no launch
    for d in (rotary_desc(B=0), rotary_desc(S=0), rotary_desc(H=0, Hk=0)):
        assert rotary(d, None, None, None, None, None, None) == OK
    assert B.workspace_size(B.ANR_OP_ROTARY, rotary_desc()) == 0


def ff_desc(**kw):
    return B.GatedFfDesc(**dict(dict(T=100, C=64, F=96, act=B.ANR_ACT_SILU, dtype=B.ANR_BF16), **kw))


def ff(d, ptrs=(P,) * 7, ws=None, size=0):
    return B.raw().anr_gated_ff(ctypes.byref(d) if d else None, *ptrs, ws, size, None)


def ff_backward(d, ptrs=(P,) * 11, ws=None, size=0):
    return B.raw().anr_gated_ff_backward(ctypes.byref(d) if d else None, *ptrs, ws, size, None)


def without(n, *gone):
    return tuple(None if i in gone else P for i in range(n))


def test_gated_ff_refusals():
    for call in (ff, ff_backward):
        assert call(None) == NULL
        for field, bad in (("T", -1), ("C", 0), ("F", 0), ("act", 5), ("act", -1), ("dtype", 3), ("dtype", -1), ("ldx", 63), ("ldy", 63), ("ldpre", 95), ("lddx", 1),
                           ("ldw", 63), ("ld_down", 95), ("lddw", 63), ("ld_ddown", -96)):
            assert call(ff_desc(**{field: bad})) == INVALID, (field, bad)
        for field, bad in (("T", 1 << 22), ("C", (1 << 20) + 1), ("F", 1 << 21), ("ldx", 1 << 22), ("ld_down", 1 << 40)):
            assert call(ff_desc(**{field: bad})) == UNSUPPORTED, (field, bad)
        assert call(ff_desc()) == WORKSPACE
    for i in range(5):
        assert ff(ff_desc(), without(7, i)) == NULL
    assert ff(ff_desc(), without(7, 5)) == NULL and ff(ff_desc(), without(7, 6)) == NULL
    for i in range(7):
        assert ff_backward(ff_desc(), without(11, i)) == NULL
        assert ff(ff_desc(), tuple(ctypes.c_void_p(0x10001) if j == i else P for j in range(7))) == INVALID
    assert ff_backward(ff_desc(), without(11, 7, 8, 9, 10)) == NULL
    assert ff(ff_desc(T=0), (None,) * 7) == OK
    for dtype in (B.ANR_F32, B.ANR_F16, B.ANR_BF16):
        for T in (1, 64, 65, 1000):
            d = ff_desc(T=T, dtype=dtype)
            for call, op in ((ff, B.ANR_OP_GATED_FF), (ff_backward, B.ANR_OP_GATED_FF_BACKWARD)):
                need = B.workspace_size(op, d)
                assert need >= T * 96 * 2
                assert call(d, ws=P, size=need - 1) == WORKSPACE and call(d, ws=ctypes.c_void_p(0x10004), size=need) == INVALID


def test_workspace_size_refuses_what_the_calls_refuse():
    for op, d in ((B.ANR_OP_GROUP_NORM, norm_desc(groups=5)), (B.ANR_OP_GROUP_NORM_BACKWARD, norm_desc(C=0)), (B.ANR_OP_ROTARY, rotary_desc(D=0)),
                  (B.ANR_OP_GATED_FF, ff_desc(C=0)), (B.ANR_OP_GATED_FF_BACKWARD, ff_desc(ldw=1)), (12, ff_desc())):
        with pytest.raises(B.AnrError):
            B.workspace_size(op, d)


def test_extents_and_strides_whose_offsets_overflow():
    """Views of more than 2^58 elements, and extents beyond the grids' and the kernels' counters, by calls and sizes alike."""
    big = [(B.ANR_OP_GROUP_NORM, norm_desc(N=1, H=1, W=1 << 29, C=4, x_stride=(1, 1, 1 << 39))),
           (B.ANR_OP_GROUP_NORM, norm_desc(N=1, H=1 << 29, W=1, C=4, y_stride=(1, 1 << 39, 1))),
           (B.ANR_OP_GROUP_NORM_BACKWARD, norm_desc(N=60000, H=1, W=1, C=4, dx_stride=((1 << 40) - 1000000, 1, 4), x_stride=(1 << 43, 1, 4))),
           (B.ANR_OP_GROUP_NORM, norm_desc(N=1, H=1 << 15, W=(1 << 15) + 1, C=4)),
           (B.ANR_OP_GROUP_NORM_BACKWARD, norm_desc(C=(1 << 20) + 4, groups=(1 << 20) + 4)),
           (B.ANR_OP_ROTARY, rotary_desc(B=1, S=(1 << 24) - 1, q_stride=(1, 1 << 39, 32))),
           (B.ANR_OP_ROTARY, rotary_desc(B=1, S=(1 << 24) - 1, pos_stride=(0, 0, 1 << 39))),
           (B.ANR_OP_ROTARY, rotary_desc(B=1 << 12, S=1 << 12))]
    for op, d in big:
        with pytest.raises(B.AnrError) as e:
            B.workspace_size(op, d)
        assert e.value.status == UNSUPPORTED, op
    assert norm(big[0][1]) == UNSUPPORTED and norm_backward(big[4][1]) == UNSUPPORTED and rotary(big[5][1]) == UNSUPPORTED
    B.workspace_size(B.ANR_OP_GROUP_NORM, norm_desc(N=1, H=1 << 15, W=1 << 15, C=4))
    B.workspace_size(B.ANR_OP_GROUP_NORM, norm_desc(C=1 << 20, groups=1 << 20))
    B.workspace_size(B.ANR_OP_ROTARY, rotary_desc(B=1, S=(1 << 24) - 1))


def test_group_norm_in_place_takes_the_same_strides():
    P2 = ctypes.c_void_p(0x20000)
    wide = (960, 240, 48)
    d = norm_desc(x_stride=wide)
    assert norm(d) == INVALID and norm(d, y=P2) == WORKSPACE
    assert norm(norm_desc(x_stride=wide, y_stride=wide)) == WORKSPACE
    assert norm_backward(d, x=P, dy=P2, dx=P) == INVALID and norm_backward(d, x=P, dy=P2, dx=P2) == WORKSPACE
    d = norm_desc(y_stride=wide)                                   # dy's
    assert norm_backward(d, x=P, dy=P2, dx=P2) == INVALID and norm_backward(d, x=P, dy=P2, dx=P) == WORKSPACE
    # the strides of single extents say nothing
    d = norm_desc(N=1, H=1, W=5, x_stride=(7, 9, 24))
    assert norm(d) == WORKSPACE


def test_binding_refuses_host_tensors_and_other_types():
    x = torch.zeros(2, 8, 3, 3).to(memory_format=torch.channels_last)
    with pytest.raises(TypeError):
        B.group_norm(x, 2, x.clone())
    with pytest.raises(TypeError):
        B.group_norm(x.double(), 2, x)
    with pytest.raises(TypeError):
        B.group_norm(x, 2, x, torch.zeros(8, dtype=torch.float16))
    with pytest.raises(TypeError):
        B.group_norm_backward(x, x, 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2), x)
    q = torch.zeros(1, 2, 3, 8)
    for pos in (torch.zeros(1, 2, dtype=torch.int64), torch.zeros(1, 2, dtype=torch.int16)):
        with pytest.raises(TypeError):
            B.rotary(q, None, pos, torch.zeros(4), q, None)
    with pytest.raises(ValueError):
        B.rotary(q, q, torch.zeros(1, 2, dtype=torch.int64), torch.zeros(4), q, None)
    m = torch.zeros(4, 4)
    with pytest.raises(TypeError):
        B.gated_ff(m, m, m, m, m)
    with pytest.raises(ValueError):
        B.gated_ff(m, m, m, m, m, gate=m)
    with pytest.raises(ValueError):
        B.gated_ff(m[0], m, m, m, m)
    with pytest.raises(TypeError):
        B.gated_ff_backward(m, m, m, m, m, m, m, m)
