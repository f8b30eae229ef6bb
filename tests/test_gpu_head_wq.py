"""4-bit weights with group scales: packing against the definition bit for bit,
and products against binary64.

Codes and the parts of x are exact, so a product is off by its sums: at most
(Kp / 16 + 8) 2^-22 sum|x w|, and its type's rounding.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 2.0 ** -126, F16: 2.0 ** -24, F32: 2.0 ** -126}


def normal(*shape, dtype=F32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def reference_pack(w, group):
    """codes [N, Kp] in [-7, 7] and scales (float32 values of bf16) of the definition."""
    n, k = w.shape
    kp = (k + 127) // 128 * 128
    v = np.zeros((n, kp), np.float32)
    v[:, :k] = w.float().cpu().numpy()
    v = v.reshape(n, -1, group)
    fine = np.isfinite(v).all(axis=2)
    top = np.where(fine, np.abs(np.where(fine[..., None], v, 0)).max(axis=2), 0).astype(np.float32)
    s = torch.from_numpy(top * (np.float32(1) / np.float32(7))).to(BF16).float().numpy()
    s = np.where((top > 0) & (s == 0), np.float32(2.0 ** -133), s)
    s = np.where(top == 0, np.float32(1), s)
    q = np.where(fine[..., None], v, 0) / s[..., None]
    whole = np.trunc(q)
    q = np.clip(whole + np.sign(q) * (np.abs(q - whole) >= 0.5), -7, 7)
    s = np.where(fine, s, np.float32(np.nan))
    return q.reshape(n, -1).astype(np.int32), s


def bytes_of(q):
    """The documented byte layout, one code at a time."""
    n, kp = q.shape
    out = np.zeros((n, kp // 2), np.uint8)
    for k in range(kp):
        at = (k // 128) * 64 + 16 * (k % 32 // 8) + 4 * (k % 128 // 32) + k % 8 // 2
        out[:, at] |= ((q[:, k] + 8) << (4 * (k % 2))).astype(np.uint8)
    return out


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N,K", [(1, 1), (5, 31), (33, 128), (20, 385), (3, 1000), (2, 4097)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_pack_and_unpack(N, K, group, dtype):
    w = normal(N, K, dtype=dtype)
    codes, scales = pvs.pvs_wq_pack(w, group)
    q, s = reference_pack(w, group)
    assert np.array_equal(scales.float().cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), bytes_of(q))
    want = (torch.from_numpy(q).float() * torch.from_numpy(s).repeat_interleave(group, dim=1))[:, :K]
    for out in (BF16, F16, F32):
        got = pvs.pvs_wq_unpack(codes, scales, group, K, out)
        assert torch.equal(got.cpu(), want.to(out))


def test_pack_zero_tiny_and_non_finite_groups():
    w = torch.zeros(6, 256, device="cuda")
    w[1, :32] = 2.0 ** -149
    w[2, 40] = float("nan")
    w[3, 255] = -math.inf
    w[4] = 3.4e38
    w[5, 0], w[5, 1:8] = 7.0, torch.arange(7, device="cuda") + 0.5   # ties
    for group in (32, 64, 128):
        codes, scales = pvs.pvs_wq_pack(w, group)
        q, s = reference_pack(w, group)
        assert np.array_equal(scales.float().cpu().numpy(), s, equal_nan=True)
        assert np.array_equal(codes.cpu().numpy(), bytes_of(q))
        y = pvs.pvs_wq_matvec(torch.ones(1, 256, device="cuda"), codes, scales, group)
        assert torch.equal(torch.isnan(y[0]).cpu(), torch.tensor([0, 0, 1, 1, 0, 0]).bool())


def check(B, N, K, group, dtype, seed=0):
    w, x = normal(N, K, dtype=dtype, seed=seed), normal(B, K, dtype=dtype, seed=seed + 1)
    codes, scales = pvs.pvs_wq_pack(w, group)
    weights = pvs.pvs_wq_unpack(codes, scales, group, K, F32).double()
    y = pvs.pvs_wq_matvec(x, codes, scales, group)
    assert y.shape == (B, N) and y.dtype == dtype
    want, size = x.double() @ weights.T, x.double().abs() @ weights.abs().T
    kp = (K + 127) // 128 * 128
    tol = (kp / 16 + 8) * 2.0 ** -22 * size + UNIT[dtype] * want.abs() + TINY[dtype]
    assert ((y.double() - want).abs() <= tol).all()
    assert torch.equal(y, pvs.pvs_wq_matvec(x, codes, scales, group))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("B,N,K", [(1, 1, 1), (1, 15, 33), (2, 16, 128), (3, 17, 129), (1, 768, 768),
                                   (5, 1000, 385), (8, 300, 1024), (9, 257, 640), (16, 40, 96)])
def test_matvec(B, N, K, group, dtype):
    check(B, N, K, group, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("B,N,K", [(1, 60_001, 256), (4, 100_000, 130), (64, 500, 200), (1, 33, 32767),
                                   (7, 5000, 12_345), (33, 20_000, 384)])
def test_matvec_long_and_many(B, N, K, dtype):
    check(B, N, K, 64, dtype, seed=3)


@pytest.mark.parametrize("dtype", [F16, F32])
def test_small_and_large_entries_of_x_keep_their_digits(dtype):
    # parts far apart, subnormals, and entries that a rounded first part would overflow
    w = torch.ones(4, 128, device="cuda")
    codes, scales = pvs.pvs_wq_pack(w, 32)
    one = pvs.pvs_wq_unpack(codes, scales, 32, 128, F32)[0, 0].double()   # 7 RN_bf16(1 / 7)
    top = torch.finfo(dtype).max
    for v in (1.0 + torch.finfo(dtype).eps, top * 0.9, torch.finfo(dtype).tiny * 1.5, -3.0):
        x = torch.zeros(1, 128, dtype=dtype, device="cuda")
        x[0, 77] = v
        y = pvs.pvs_wq_matvec(x, codes, scales, 32).double()
        want = (x[0, 77].double() * one).to(dtype).double()
        assert ((y - want).abs() <= 2.0 ** -22 * want.abs() + TINY[dtype]).all(), v


def test_non_finite_x_reaches_the_products():
    w = normal(40, 200)
    codes, scales = pvs.pvs_wq_pack(w, 64)
    x = normal(3, 200, seed=1)
    x[1, 5] = float("nan")
    y = pvs.pvs_wq_matvec(x, codes, scales, 64)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


def test_strided_operands_and_views():
    w = normal(90, 300, seed=2)
    codes, scales = pvs.pvs_wq_pack(w[:, 10:260], 32)
    same = pvs.pvs_wq_pack(w[:, 10:260].contiguous(), 32)
    assert torch.equal(codes, same[0]) and torch.equal(scales, same[1])
    x = normal(4, 600, seed=3)
    want = pvs.pvs_wq_matvec(x[:, 1:251].contiguous(), codes, scales, 32)
    assert torch.equal(pvs.pvs_wq_matvec(x[:, 1:251], codes, scales, 32), want)
    room = torch.zeros(1 + codes.numel(), dtype=torch.uint8, device="cuda")
    room[1:] = codes.reshape(-1)
    odd = room[1:].view(codes.shape)
    assert torch.equal(pvs.pvs_wq_matvec(x[:, 1:251], odd, scales, 32), want)
    assert torch.equal(pvs.pvs_wq_matvec(x[:, 1:251], codes[30:], scales[30:], 32), want[:, 30:])


def test_offsets_past_32_bits():
    N, K = 6_000_000, 1536
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    codes[codes & 15 == 0] += 8            # a code is 1 .. 15
    codes[codes < 16] += 128
    scales = torch.ones(N, K // 128, dtype=BF16, device="cuda")
    x = normal(2, K, seed=4)
    y = pvs.pvs_wq_matvec(x, codes, scales, 128)
    tail = slice(N - 3000, N)
    weights = pvs.pvs_wq_unpack(codes[tail], scales[tail], 128, K, F32).double()
    want, size = x.double() @ weights.T, x.double().abs() @ weights.abs().T
    assert ((y[:, tail].double() - want).abs() <= (K / 16 + 8) * 2.0 ** -22 * size).all()


def test_streams_graphs_and_nothing():
    w, x = normal(700, 500, dtype=BF16), normal(2, 500, dtype=BF16, seed=1)
    codes, scales = pvs.pvs_wq_pack(w, 64)
    want = pvs.pvs_wq_matvec(x, codes, scales, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = pvs.pvs_wq_matvec(x, codes, scales, 64)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pvs.pvs_wq_matvec(x, codes, scales, 64)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert pvs.pvs_wq_matvec(x[:0], codes, scales, 64).shape == (0, 700)
    assert pvs.pvs_wq_matvec(x, codes[:0], scales[:0], 64).shape == (2, 0)
    assert pvs.pvs_wq_pack(w[:0], 64)[0].shape == (0, 256)


def test_refusals():
    w, x = normal(10, 200), normal(2, 200)
    codes, scales = pvs.pvs_wq_pack(w, 32)
    for exc, f, args in [
            (ValueError, pvs.pvs_wq_pack, (w, 16)), (TypeError, pvs.pvs_wq_pack, (w.double(), 32)),
            (TypeError, pvs.pvs_wq_pack, (w.cpu(), 32)), (ValueError, pvs.pvs_wq_pack, (w[0], 32)),
            (ValueError, pvs.pvs_wq_matvec, (x, codes, scales, 48)),
            (ValueError, pvs.pvs_wq_matvec, (x, codes, scales, 64)),
            (ValueError, pvs.pvs_wq_matvec, (x[:, :100], codes, scales, 32)),
            (ValueError, pvs.pvs_wq_matvec, (x[0], codes, scales, 32)),
            (ValueError, pvs.pvs_wq_matvec, (normal(65, 200), codes, scales, 32)),
            (TypeError, pvs.pvs_wq_matvec, (x, codes.int(), scales, 32)),
            (TypeError, pvs.pvs_wq_matvec, (x, codes, scales.float(), 32)),
            (ValueError, pvs.pvs_wq_matvec, (x, codes[:, :63], scales, 32)),
            (ValueError, pvs.pvs_wq_unpack, (codes, scales, 32, 100, F32)),
            (TypeError, pvs.pvs_wq_unpack, (codes, scales, 32, 200, torch.float64))]:
        with pytest.raises(exc):
            f(*args)
