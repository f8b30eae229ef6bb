"""The refusals of table lookups, distillation and microscaled rows at the C boundary, which
come before any CUDA call."""
import ctypes

import pytest

import paper_2608_07152_gb300 as pvs

L = pvs._lib
P = 1 << 20                       # a pointer that nothing reads
BAD = pvs.PVS_ERR_INVALID


def lookup(**kw):
    a = dict(w=P, ldw=16, items=9, dim=16, dtype=0, ids=P, rows=4, scale=1.0, ignore=-100, y=P, ldy=16, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return L.pvs_embed_forward(*a.values())


def gradient(**kw):
    a = dict(dy=P, lddy=16, ids=P, rows=4, items=9, dim=16, dtype=0, scale=1.0, ignore=-100, dw=P, lddw=16, ws=P,
             bytes=1 << 20, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return L.pvs_embed_backward(*a.values())


SHAPES = [dict(rows=-1), dict(rows=1 << 31), dict(items=0), dict(items=1 << 31), dict(dim=0),
          dict(dtype=3), dict(dtype=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(ids=None),
          dict(ids=P + 4)]


@pytest.mark.parametrize("bad", SHAPES + [dict(w=None), dict(w=P + 1), dict(y=None), dict(y=P + 1), dict(ldw=15),
                                          dict(ldy=15), dict(dim=32768, ldw=40000, ldy=40000),
                                          dict(dtype=2, w=P + 2), dict(dtype=2, y=P + 2)])
def test_lookup_refusals(bad):
    assert lookup(**bad) == BAD


@pytest.mark.parametrize("bad", SHAPES + [dict(dy=None), dict(dy=P + 1), dict(dw=None), dict(dw=P + 1), dict(lddy=15),
                                          dict(lddw=15), dict(dim=32768, lddy=40000, lddw=40000), dict(bytes=31),
                                          dict(ws=None), dict(ws=P + 128)])
def test_gradient_refusals(bad):
    assert gradient(**bad) == BAD


def test_lookup_of_nothing():
    assert lookup(rows=0, w=None, ids=None, y=None) == pvs.PVS_OK
    n = ctypes.c_size_t(7)
    assert L.pvs_embed_workspace(0, 9, 16, ctypes.byref(n)) == pvs.PVS_OK and n.value == 0
    assert L.pvs_embed_workspace(4, 9, 16, None) == BAD
    assert L.pvs_embed_workspace(4, 0, 16, ctypes.byref(n)) == BAD


@pytest.mark.parametrize("rows", [1, 32, 33, 8192, 8193, 100_000, 1 << 30])
def test_gradient_workspace(rows):
    # the documented most; each of eight parts may be rounded up to 256 bytes, and totals take 4 KB
    for items, dim in ((1, 1), (1000, 385), (1 << 20, 4096), ((1 << 31) - (1 << 16), 32767)):
        n = ctypes.c_size_t()
        assert L.pvs_embed_workspace(rows, items, dim, ctypes.byref(n)) == pvs.PVS_OK
        padded = (dim + 7) // 8 * 8
        piece = 8 if rows * ((dim + 255) // 256) < 38_912 else 32
        pieces = (rows + piece - 1) // piece
        tiles = (rows + 1023) // 1024
        assert 8 * rows <= n.value <= 16 * rows + pieces * (8 * padded + 4) + 4096 * (tiles + 1) + 8 * 256


def distill(student=None, **kw):
    s = dict(x=P, w=P, targets=None, bias=None, rows=4, items=9, ldx=16, ldw=16, ignore_index=-100, dim=16,
             dtype=pvs.PVS_BF16, scale=1.0, reserved=0)
    s.update(student or {})
    a = dict(ids=P, logits=P, top=5, teacher_dtype=pvs.PVS_F32, teacher_scale=1.0, reserved=0)
    a.update(kw)
    return pvs.pvs_distill_args(pvs.pvs_xent_args(*s.values()), *a.values())


@pytest.mark.parametrize("bad", [
    dict(top=0), dict(top=1025), dict(teacher_dtype=3), dict(teacher_dtype=-1), dict(teacher_scale=0.0),
    dict(teacher_scale=float("nan")), dict(teacher_scale=float("inf")), dict(reserved=1), dict(ids=None),
    dict(ids=P + 4), dict(student=dict(rows=-1)), dict(student=dict(items=0)), dict(student=dict(scale=-1.0)),
    dict(student=dict(ldx=15)), dict(student=dict(x=None)), dict(student=dict(w=P + 1)), dict(student=dict(reserved=1)),
    dict(student=dict(bias=P + 2))])
def test_distill_refusals(bad):
    a = distill(**bad)
    n = ctypes.c_size_t()
    assert L.pvs_distill_workspace(ctypes.byref(a), 0, ctypes.byref(n)) == BAD
    assert L.pvs_distill_forward(ctypes.byref(a), P, P, P, P, 0, None) == BAD
    assert L.pvs_distill_backward(ctypes.byref(a), P, P, P, P, 16, P, 16, P, 0, None) == BAD


def test_distill_pointers():
    n = ctypes.c_size_t()
    a = distill()
    assert L.pvs_distill_workspace(None, 0, ctypes.byref(n)) == BAD
    assert L.pvs_distill_workspace(ctypes.byref(a), 0, None) == BAD
    for bad in ((None, P, P), (P, None, P), (P, P, None), (P + 2, P, P), (P, P + 8, P), (P, P, P + 2)):
        assert L.pvs_distill_forward(ctypes.byref(a), *bad, P, 0, None) == BAD
    for a2 in (distill(logits=None), distill(logits=P + 2)):
        assert L.pvs_distill_forward(ctypes.byref(a2), P, P, P, P, 0, None) == BAD
    for bad in ((None, P, P, P, 16, P, 16), (P, None, P, P, 16, P, 16), (P, P, None, P, 16, P, 16),
                (P + 8, P, P, P, 16, P, 16), (P, P + 2, P, P, 16, P, 16), (P, P, P, P + 1, 16, P, 16),
                (P, P, P, P, 15, P, 16), (P, P, P, P, 16, P, 15), (P, P, P, P, 16, P + 1, 16)):
        assert L.pvs_distill_backward(ctypes.byref(a), *bad, P, 0, None) == BAD
    none = distill(student=dict(rows=0, x=None), ids=None, logits=None)
    assert L.pvs_distill_forward(ctypes.byref(none), None, None, None, None, 0, None) == pvs.PVS_OK
    assert L.pvs_distill_backward(ctypes.byref(none), None, None, None, P, 16, None, 16, None, 0, None) == pvs.PVS_OK


def test_distill_layout(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f for f, _ in pvs.pvs_distill_args._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"head.h\"\nint main(void) {\n"
                   + 'printf("%zu\\n", sizeof(pvs_distill_args));\n'
                   + "".join(f'printf("%zu\\n", offsetof(pvs_distill_args, {n}));\n' for n in names) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(pvs.pvs_distill_args)] + [getattr(pvs.pvs_distill_args, n).offset for n in names]


def pack(**kw):
    a = dict(x=P, ldx=300, rows=4, cols=300, dtype=0, group=16, codes=P, scales=P, row_scales=P, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return L.pvs_mx_pack(*a.values())


def unpack(**kw):
    a = dict(codes=P, scales=P, row_scales=P, rows=4, cols=300, group=16, out=P, ldout=300, dtype=0, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return L.pvs_mx_unpack(*a.values())


def product(**kw):
    a = dict(x=P, ldx=300, batch=3, codes=P, scales=P, row_scales=P, rows=4, cols=300, group=16, dtype=0, y=P, ldy=4,
             ws=P, bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return L.pvs_mx_matmul(*a.values())


OPERAND = [dict(codes=None), dict(codes=P + 8), dict(scales=None), dict(scales=P + 8), dict(row_scales=None),
           dict(row_scales=P + 2), dict(group=8), dict(group=64), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
           dict(dtype=3), dict(dtype=-1)]


@pytest.mark.parametrize("bad", OPERAND + [dict(x=None), dict(x=P + 1), dict(ldx=299), dict(cols=32768, ldx=40000)])
def test_mx_pack_refusals(bad):
    assert pack(**bad) == BAD


@pytest.mark.parametrize("bad", OPERAND + [dict(out=None), dict(out=P + 1), dict(ldout=299), dict(cols=32768, ldout=40000)])
def test_mx_unpack_refusals(bad):
    assert unpack(**bad) == BAD


@pytest.mark.parametrize("bad", OPERAND + [dict(x=None), dict(x=P + 1), dict(y=None), dict(y=P + 1), dict(ldx=299),
                                           dict(ldy=3), dict(batch=-1), dict(batch=1 << 31),
                                           dict(cols=32768, ldx=40000)])
def test_mx_matmul_refusals(bad):
    assert product(**bad) == BAD


def test_mx_of_nothing():
    assert pack(rows=0, x=None, codes=None, scales=None, row_scales=None) == pvs.PVS_OK
    assert unpack(rows=0, out=None, codes=None, scales=None, row_scales=None) == pvs.PVS_OK
    assert product(batch=0, x=None, y=None, codes=None, scales=None, row_scales=None, ws=None) == pvs.PVS_OK
    assert product(rows=0, ldy=0, codes=None, scales=None, row_scales=None, ws=None) == pvs.PVS_OK
    n = ctypes.c_size_t(3)
    assert L.pvs_mx_workspace(0, 5, 128, 16, ctypes.byref(n)) == pvs.PVS_OK and n.value == 0
    assert L.pvs_mx_workspace(5, 5, 128, 16, None) == BAD
    assert L.pvs_mx_workspace(5, 5, 128, 8, ctypes.byref(n)) == BAD
