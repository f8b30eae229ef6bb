"""include/head.h at the C boundary without a GPU: the argument structure's layout,
and the refusals that come before any CUDA call."""
import ctypes
import os
import subprocess

import pytest

import paper_2608_07152_gb300 as pvs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = pvs._lib
P = 1 << 20                       # a pointer that nothing reads


def args(**kw):
    a = dict(x=P, w=P, targets=P, bias=None, rows=4, items=9, ldx=16, ldw=16, ignore_index=-100,
             dim=16, dtype=pvs.PVS_BF16, scale=1.0, reserved=0)
    a.update(kw)
    return pvs.pvs_xent_args(*[a[f] for f, _ in pvs.pvs_xent_args._fields_])


def test_argument_layout(tmp_path):
    names = [f for f, _ in pvs.pvs_xent_args._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"head.h\"\nint main(void) {\n"
                   + 'printf("%zu\\n", sizeof(pvs_xent_args));\n'
                   + "".join(f'printf("%zu\\n", offsetof(pvs_xent_args, {n}));\n' for n in names)
                   + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [ctypes.sizeof(pvs.pvs_xent_args)] + [getattr(pvs.pvs_xent_args, n).offset
                                                        for n in names]


def test_entry_points_are_exported():
    for name in pvs._head.EXPORTED:
        assert hasattr(L, name) and name in pvs.EXPORTED and callable(getattr(pvs, name, None)) or \
            name.endswith("_workspace"), name


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=1 << 31), dict(items=0), dict(items=1 << 31), dict(dim=0),
    dict(dim=40000, ldx=40000, ldw=40000), dict(dtype=3), dict(dtype=-1), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(reserved=1),
    dict(ldx=15), dict(ldw=8), dict(x=None), dict(w=None), dict(targets=None)])
def test_xent_refusals(bad):
    a = args(**bad)
    n = ctypes.c_size_t()
    assert L.pvs_xent_workspace(ctypes.byref(a), 1, ctypes.byref(n)) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_forward(ctypes.byref(a), P, P, P, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_backward(ctypes.byref(a), P, P, P, 16, P, 16, P, 0, None) == pvs.PVS_ERR_INVALID


def test_xent_null_arguments():
    a = args()
    n = ctypes.c_size_t()
    assert L.pvs_xent_workspace(None, 0, ctypes.byref(n)) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_workspace(ctypes.byref(a), 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_forward(ctypes.byref(a), None, P, P, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_forward(ctypes.byref(a), P, P + 4, P, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_xent_backward(ctypes.byref(a), None, P, P, 16, P, 16, P, 0, None) == \
        pvs.PVS_ERR_INVALID
    assert L.pvs_xent_backward(ctypes.byref(a), P, P, P, 15, P, 16, P, 0, None) == \
        pvs.PVS_ERR_INVALID
    none = args(rows=0, x=None, targets=None)
    assert L.pvs_xent_forward(ctypes.byref(none), None, None, None, 0, None) == pvs.PVS_OK


def test_ckpt_refusals():
    store = lambda r=3, k=8, t=0, act=0, ldx=8, ldc=8, x=P, c=P, s=P, y=None, ldy=8: \
        L.pvs_ckpt_store(x, ldx, r, k, t, act, c, ldc, s, y, ldy, None)   # noqa: E731
    for kw in (dict(r=-1), dict(k=0), dict(k=32768, ldx=40000, ldc=40000), dict(t=3), dict(act=2),
               dict(act=1), dict(ldx=7), dict(ldc=7), dict(x=None), dict(c=None), dict(s=None),
               dict(act=1, y=P, ldy=7)):
        assert store(**kw) == pvs.PVS_ERR_INVALID, kw
    assert store(r=0, x=None, c=None, s=None) == pvs.PVS_OK
    assert L.pvs_ckpt_load(P, 8, P, 3, 8, None, 8, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_load(P, 7, P, 3, 8, P, 8, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_act_backward(P, 8, P, 8, P, 3, 8, 0, 0, P, 8, None) == pvs.PVS_ERR_INVALID
    n = ctypes.c_size_t()
    assert L.pvs_ckpt_grad_workspace(3, 0, 8, 0, ctypes.byref(n)) == pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_grad_workspace(3, 8, 8, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_grad_weight(P, 7, P, 8, P, 3, 8, 8, 0, P, 8, P, 1 << 30, None) == \
        pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_grad_weight(P, 8, P, 8, P, 3, 8, 8, 0, None, 8, P, 1 << 30, None) == \
        pvs.PVS_ERR_INVALID


def test_wq_refusals():
    assert L.pvs_wq_pack(P, 8, 3, 8, 0, 16, P, P, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_pack(P, 7, 3, 8, 0, 32, P, P, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_pack(P, 8, 3, 8, 0, 32, P + 1, P, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_unpack(P, P + 2, 3, 8, 32, P, 8, 0, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(P, 8, 65, P, P, 3, 8, 32, 0, P, 3, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(P, 8, 1, P, P, 3, 8, 32, 0, P, 2, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(None, 8, 1, P, P, 3, 8, 32, 0, P, 3, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(None, 8, 0, None, None, 3, 8, 32, 0, None, 3, None) == pvs.PVS_OK
