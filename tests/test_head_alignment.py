"""Pointers that are not aligned to their elements are refused at the C boundary, before
any CUDA call: the kernels would read and write them misaligned."""
import ctypes

import pytest

import paper_2608_07152_gb300 as pvs

torch = pytest.importorskip("torch")
# (were a call not refused, a GPU would read what the pointers say)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="pointers that nothing may read")

L = pvs._lib
P = 1 << 20                       # a pointer that nothing reads
SIZE = {pvs.PVS_BF16: 2, pvs.PVS_F16: 2, pvs.PVS_F32: 4}


def off(value, name, bad, by):
    return value + by if name == bad else value


@pytest.mark.parametrize("dtype", SIZE)
@pytest.mark.parametrize("bad", ["x", "w", "targets", "bias", "loss", "grad_loss", "dx", "dw"])
def test_xent(bad, dtype):
    by = {"targets": 4, "bias": 2, "loss": 2, "grad_loss": 2}.get(bad, SIZE[dtype] // 2)
    p = {n: off(P, n, bad, by) for n in ("x", "w", "targets", "bias", "loss", "grad_loss", "dx", "dw")}
    a = pvs.pvs_xent_args(p["x"], p["w"], p["targets"], p["bias"], 40, 9, 16, 16, -100, 16, dtype, 1.0, 0)
    if bad in ("x", "w", "targets", "bias"):
        n = ctypes.c_size_t()
        assert L.pvs_xent_workspace(ctypes.byref(a), 0, ctypes.byref(n)) == pvs.PVS_ERR_INVALID
    if bad in ("x", "w", "targets", "bias", "loss"):
        assert L.pvs_xent_forward(ctypes.byref(a), p["loss"], P, P, 0, None) == pvs.PVS_ERR_INVALID
    if bad != "loss":
        assert L.pvs_xent_backward(ctypes.byref(a), P, p["grad_loss"], p["dx"], 16, p["dw"], 16, P, 0,
                                   None) == pvs.PVS_ERR_INVALID


@pytest.mark.parametrize("dtype", SIZE)
def test_gradient_of_no_rows(dtype):
    a = pvs.pvs_xent_args(None, P, None, None, 0, 9, 16, 16, -100, 16, dtype, 1.0, 0)
    assert L.pvs_xent_backward(ctypes.byref(a), None, None, None, 16, P + SIZE[dtype] // 2, 16, None, 0,
                               None) == pvs.PVS_ERR_INVALID


@pytest.mark.parametrize("dtype", SIZE)
def test_ckpt(dtype):
    h = SIZE[dtype] // 2
    for x, s, y in ((P + h, P, P), (P, P + 2, P), (P, P, P + h)):
        assert L.pvs_ckpt_store(x, 8, 3, 8, dtype, 1, P, 8, s, y, 8, None) == pvs.PVS_ERR_INVALID
    for s, out in ((P + 2, P), (P, P + h)):
        assert L.pvs_ckpt_load(P, 8, s, 3, 8, out, 8, dtype, None) == pvs.PVS_ERR_INVALID
    for dy, s, dx in ((P + h, P, P), (P, P + 2, P), (P, P, P + h)):
        assert L.pvs_ckpt_act_backward(dy, 8, P, 8, s, 3, 8, dtype, 1, dx, 8, None) == pvs.PVS_ERR_INVALID
        assert L.pvs_ckpt_grad_weight(dy, 8, P, 8, s, 3, 8, 8, dtype, dx, 8, P, 0, None) == \
            pvs.PVS_ERR_INVALID
    assert L.pvs_ckpt_grad_weight(None, 8, None, 8, None, 0, 8, 8, dtype, P + h, 8, None, 0, None) == \
        pvs.PVS_ERR_INVALID


@pytest.mark.parametrize("dtype", SIZE)
def test_wq(dtype):
    h = SIZE[dtype] // 2
    assert L.pvs_wq_pack(P + h, 8, 3, 8, dtype, 32, P, P, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_unpack(P, P, 3, 8, 32, P + h, 8, dtype, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(P + h, 8, 1, P, P, 3, 8, 32, dtype, P, 3, None) == pvs.PVS_ERR_INVALID
    assert L.pvs_wq_matvec(P, 8, 1, P, P, 3, 8, 32, dtype, P + h, 3, None) == pvs.PVS_ERR_INVALID
