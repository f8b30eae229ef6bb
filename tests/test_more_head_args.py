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


@pytest.mark.parametrize("rows", [1, 32, 33, 4096, 4097, 100_000, 1 << 30])
def test_gradient_workspace(rows):
    # the documented most; each of seven parts may be rounded up to 256 bytes, and totals take 4 KB
    for items, dim in ((1, 1), (1000, 385), (1 << 20, 4096), ((1 << 31) - (1 << 16), 32767)):
        n = ctypes.c_size_t()
        assert L.pvs_embed_workspace(rows, items, dim, ctypes.byref(n)) == pvs.PVS_OK
        padded = (dim + 7) // 8 * 8
        pieces = (rows + 31) // 32
        tiles = (rows + 2047) // 2048
        assert 8 * rows <= n.value <= 16 * rows + 8 * pieces * padded + 4096 * (tiles + 1) + 7 * 256
