"""Rows kept in 8 bits and the backward steps that read them, against the
quantizer's definition and binary64.

Codes and scales are compared bit for bit with the definition.  A GELU in float32
is off by at most 2^-21 max(|x|, 1), a slope by 2^-20 (1 + |x|); a weight gradient by
its operand's rounding (one bf16: 2^-8; f16 in two parts: 2^-16; float32 in three:
2^-24) and (R / 16 + 8) 2^-23 through sum|dy x|, and its type's rounding.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
OPERAND = {BF16: 2.0 ** -8, F16: 2.0 ** -15, F32: 2.0 ** -23}
TINY = {BF16: 2.0 ** -126, F16: 2.0 ** -24, F32: 2.0 ** -126}


def rows(r, k, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(r, k, generator=g, device="cuda")
    return (x * torch.exp(spread * torch.randn(r, 1, generator=g, device="cuda"))).to(dtype)


def quantized(x):
    """Scales and codes of the definition, in numpy."""
    v = x.float().cpu().numpy()
    s = np.ones(v.shape[0], np.float32)
    z = np.zeros(v.shape, np.int8)
    for i, row in enumerate(v):
        if not np.isfinite(row).all():
            s[i] = np.nan
            continue
        top = np.abs(row).max()
        if top > 0:
            s[i] = np.float32(top) * (np.float32(1) / np.float32(127))
            if s[i] == 0:
                s[i] = np.float32(2.0 ** -149)
            q = row / s[i]
            whole = np.trunc(q)
            q = whole + np.sign(q) * (np.abs(q - whole) >= 0.5)
            z[i] = np.clip(q, -127, 127).astype(np.int8)
    return z, s


def gelu(x):
    return 0.5 * x * torch.erfc(-x / math.sqrt(2.0))


def slope(x):
    return (0.5 * torch.erfc(-x / math.sqrt(2.0))
            + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi))


SHAPES = [(1, 1), (3, 5), (7, 31), (4, 32), (5, 33), (65, 128), (33, 385), (17, 768), (1001, 1536),
          (9, 2048), (3, 2049), (2, 8191), (2, 32767)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,K", SHAPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_store_and_load(R, K, dtype, act):
    x = rows(R, K, dtype)
    code = pvs.PVS_ACT_GELU if act == "gelu" else pvs.PVS_ACT_NONE
    codes, scales, y = pvs.pvs_ckpt_store(x, act=code)
    z, s = quantized(x)
    assert np.array_equal(scales.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), z)
    if act == "none":
        assert y is None
    else:
        want = gelu(x.double())
        tol = 2.0 ** -21 * x.double().abs().clamp(min=1.0) + UNIT[dtype] * want.abs() + TINY[dtype]
        assert ((y.double() - want).abs() <= tol).all()
    for out in (BF16, F16, F32):
        kept = pvs.pvs_ckpt_load(codes, scales, out)
        assert torch.equal(kept, (codes.float() * scales[:, None]).to(out))


def test_ties_zero_tiny_and_non_finite_rows():
    x = torch.zeros(9, 40, device="cuda")
    x[1] = 127.0
    x[1, 1:20] = torch.arange(1, 20, device="cuda") - 0.5          # ties, half away from zero
    x[1, 20:39] = -(torch.arange(1, 20, device="cuda") - 0.5)
    x[2, 3] = 2.0 ** -149
    x[3] = torch.arange(40, device="cuda") * 2.0 ** -140
    x[4, 0], x[4, 1] = 3.0e38, -3.4e38
    x[5, 7] = float("nan")
    x[6, 39] = math.inf
    x[7, 0] = -math.inf
    x[8] = -1e-30
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    z, s = quantized(x)
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), z)
    kept = pvs.pvs_ckpt_load(codes, scales, F32)
    assert torch.isnan(kept[5:8]).all() and torch.isfinite(kept[:5]).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,K", [(1, 1), (5, 33), (70, 385), (300, 768), (2, 8191)])
def test_act_backward(R, K, dtype):
    x, dy = rows(R, K, dtype, 1), rows(R, K, dtype, 2)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    dx = pvs.pvs_ckpt_act_backward(dy, codes, scales, pvs.PVS_ACT_GELU)
    kept = (codes.float() * scales[:, None]).double()
    want = dy.double() * slope(kept)
    tol = (2.0 ** -20 * (1 + kept.abs()) * dy.double().abs() + UNIT[dtype] * want.abs()
           + TINY[dtype])
    assert ((dx.double() - want).abs() <= tol).all()


def test_act_backward_against_differences():
    # y(x + h) - y(x - h) over 2 h of the activation that store computes: each y is
    # off by 2^-21 max(|x|, 1), the GELU's third derivative is at most 1
    x = rows(50, 96, F32, 3)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    kept = pvs.pvs_ckpt_load(codes, scales, F32)
    h = 2.0 ** -6
    up = pvs.pvs_ckpt_store(kept + h, act=pvs.PVS_ACT_GELU)[2].double()
    down = pvs.pvs_ckpt_store(kept - h, act=pvs.PVS_ACT_GELU)[2].double()
    step = (kept + h).double() - (kept - h).double()
    one = pvs.pvs_ckpt_act_backward(torch.ones_like(kept), codes, scales, pvs.PVS_ACT_GELU).double()
    k = kept.double().abs()
    tol = (4 * 2.0 ** -21 * (k + 1) + 2.0 ** -23 * k) / (2 * h) + h * h / 6 + 2.0 ** -20 * (1 + k)
    assert ((up - down) / step - one).abs().le(tol).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,N,K", [(1, 1, 1), (1, 300, 40), (7, 9, 17), (64, 128, 256),
                                   (65, 129, 257), (1000, 385, 770), (5000, 100, 1000),
                                   (20_011, 64, 72), (300, 2050, 1100)])
def test_grad_weight(R, N, K, dtype):
    x, dy = rows(R, K, dtype, 4, spread=0.5), rows(R, N, dtype, 5, spread=0.5)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    assert dw.dtype == dtype and dw.shape == (N, K)
    kept = codes.double() * scales.double()[:, None]
    want = dy.double().T @ kept
    size = dy.double().abs().T @ kept.abs()
    tol = ((OPERAND[dtype] + (R / 16 + 8) * 2.0 ** -23) * size + UNIT[dtype] * want.abs()
           + TINY[dtype])
    assert ((dw.double() - want).abs() <= tol).all()
    assert torch.equal(dw, pvs.pvs_ckpt_grad_weight(dy, codes, scales))
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK


def test_grad_weight_by_differences():
    # the layer is linear in its weights: the loss <dy, x W^T> along a direction
    x, dy = rows(200, 70, F32, 6), rows(200, 50, F32, 7)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    kept = pvs.pvs_ckpt_load(codes, scales, F32).double()
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales).double()
    v = rows(50, 70, F32, 8).double()
    loss = lambda w: (dy.double() * (kept @ w.T)).sum()   # noqa: E731
    diff = (loss(v) - loss(-v)) / 2
    size = (v.abs() * (dy.double().abs().T @ kept.abs())).sum()
    assert abs(diff - (dw * v).sum()) <= (200 / 16 + 8) * 2.0 ** -22 * size


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_operands(dtype):
    wide = rows(60, 300, dtype, 9)
    x, dy = wide[:, 3:200], rows(60, 300, dtype, 10)[:, 1:198]
    codes, scales, y = pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU)
    same = pvs.pvs_ckpt_store(x.contiguous(), act=pvs.PVS_ACT_GELU)
    assert torch.equal(codes, same[0]) and torch.equal(scales, same[1]) and torch.equal(y, same[2])
    room = torch.zeros(60, 333, dtype=torch.int8, device="cuda")
    room[:, 5:202] = codes
    c = room[:, 5:202]
    assert torch.equal(pvs.pvs_ckpt_load(c, scales, dtype), pvs.pvs_ckpt_load(codes, scales, dtype))
    assert torch.equal(pvs.pvs_ckpt_act_backward(dy, c, scales),
                       pvs.pvs_ckpt_act_backward(dy.contiguous(), codes, scales))
    assert torch.equal(pvs.pvs_ckpt_grad_weight(dy, c, scales),
                       pvs.pvs_ckpt_grad_weight(dy.contiguous(), codes, scales))
    t = x.T.contiguous().T
    assert torch.equal(pvs.pvs_ckpt_store(t)[0], codes)
    assert torch.equal(pvs.pvs_ckpt_store(x[::3])[0], codes[::3])


def test_rows_that_hold_nan_reach_what_they_touch():
    x, dy = rows(10, 40, F32, 11), rows(10, 30, F32, 12)
    x[4, 7] = float("nan")
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    assert torch.isnan(pvs.pvs_ckpt_grad_weight(dy, codes, scales)).all()
    dx = pvs.pvs_ckpt_act_backward(dy[:, :1].expand(10, 40).contiguous(), codes, scales)
    assert torch.equal(torch.isnan(dx).any(dim=1), torch.arange(10, device="cuda") == 4)


def test_offsets_past_32_bits():
    R, K = 1_060_000, 2048
    x = torch.empty(R, K, dtype=BF16, device="cuda")
    for i in range(0, R, 1 << 17):
        x[i:i + (1 << 17)] = torch.randn(min(1 << 17, R - i), K, device="cuda")
    codes, scales, y = pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU)
    tail = slice(R - 500, R)
    c2, s2, y2 = pvs.pvs_ckpt_store(x[tail], act=pvs.PVS_ACT_GELU)
    assert torch.equal(codes[tail], c2) and torch.equal(scales[tail], s2)
    assert torch.equal(y[tail], y2)
    assert torch.equal(pvs.pvs_ckpt_load(codes, scales, BF16)[tail],
                       pvs.pvs_ckpt_load(c2, s2, BF16))
    assert torch.equal(pvs.pvs_ckpt_act_backward(x, codes, scales)[tail],
                       pvs.pvs_ckpt_act_backward(x[tail], c2, s2))
    # a weight gradient over the same rows: only the last ones count
    dy = torch.zeros(R, 8, dtype=BF16, device="cuda")
    dy[tail] = 1.0
    want = (codes[tail].double() * scales[tail].double()[:, None]).sum(dim=0)
    size = (codes[tail].double() * scales[tail].double()[:, None]).abs().sum(dim=0)
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales).double()
    tol = (2.0 ** -8 + (R / 16 + 8) * 2.0 ** -23) * size + 2.0 ** -8 * want.abs()
    assert ((dw - want).abs() <= tol).all()


def test_streams_graphs_and_no_rows():
    x, dy = rows(300, 200, BF16, 13), rows(300, 120, BF16, 14)

    def run():
        codes, scales, y = pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU)
        return codes, scales, y, pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    codes, scales, y = pvs.pvs_ckpt_store(x[:0], act=pvs.PVS_ACT_GELU)
    assert codes.shape == (0, 200) and y.shape == (0, 200)
    dw = pvs.pvs_ckpt_grad_weight(dy[:0], codes, scales)
    assert dw.shape == (120, 200) and not dw.any()


def test_refusals():
    x = rows(6, 20, BF16)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    for exc, f, args in [
            (TypeError, pvs.pvs_ckpt_store, (x.cpu(),)), (TypeError, pvs.pvs_ckpt_store, (x.double(),)),
            (ValueError, pvs.pvs_ckpt_store, (x[0],)), (ValueError, pvs.pvs_ckpt_store, (x[:, :0],)),
            (pvs.PvsError, pvs.pvs_ckpt_store, (x, 9)),
            (TypeError, pvs.pvs_ckpt_load, (codes.int(), scales, BF16)),
            (TypeError, pvs.pvs_ckpt_load, (codes, scales, torch.float64)),
            (TypeError, pvs.pvs_ckpt_load, (codes, scales.half(), BF16)),
            (ValueError, pvs.pvs_ckpt_load, (codes, scales[:3], BF16)),
            (ValueError, pvs.pvs_ckpt_act_backward, (x[:, :5], codes, scales)),
            (pvs.PvsError, pvs.pvs_ckpt_act_backward, (x, codes, scales, pvs.PVS_ACT_NONE)),
            (ValueError, pvs.pvs_ckpt_grad_weight, (x[:4], codes, scales)),
            (TypeError, pvs.pvs_ckpt_grad_weight, (x.int(), codes, scales))]:
        with pytest.raises(exc):
            f(*args)
