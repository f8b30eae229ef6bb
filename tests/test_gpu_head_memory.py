"""What the head's operators want of memory beside their operands and results, and calls
that are cut into pieces for it."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_ckpt import OPERAND  # noqa: E402
from test_gpu_head_xent import BF16, F16, F32, UNIT, close  # noqa: E402

pytestmark = pytest.mark.gpu

GB = 1 << 30


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,N,K", [(262_144, 8192, 8192), (2_000_000_000, 1024, 1024), (1 << 20, 32, 32767)])
def test_weight_gradients_scratch_is_bounded(R, N, K, dtype):
    # copies of a piece of the rows, and float32 sums
    size = ctypes.c_size_t()
    code = {BF16: pvs.PVS_BF16, F16: pvs.PVS_F16, F32: pvs.PVS_F32}[dtype]
    assert pvs._lib.pvs_ckpt_grad_workspace(R, N, K, code, ctypes.byref(size)) == pvs.PVS_OK
    assert size.value <= 3 * GB + GB // 4


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("strided", [False, True])
def test_weight_gradient_in_pieces_of_rows(dtype, strided):
    # more than 1 GB of copies; of one sign, so that every piece counts in every entry
    R, N, K = 300_001, 64, 2056
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.rand(R, K, generator=g, device="cuda").to(dtype)
    dy = (torch.rand(R, N + strided, generator=g, device="cuda") / 256).to(dtype)[:, strided:]
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    del x
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    want = torch.zeros(N, K, dtype=torch.float64, device="cuda")
    for i in range(0, R, 1 << 16):
        at = slice(i, i + (1 << 16))
        want += dy[at].double().T @ (codes[at].double() * scales[at].double()[:, None])
    close(dw, want, (OPERAND[dtype] + (R / 16 + 8) * 2.0 ** -23 + UNIT[dtype]) * want)


def xent_args(rows, items, dim, dtype):
    p = 1 << 20                    # a pointer that nothing reads
    code = {BF16: pvs.PVS_BF16, F16: pvs.PVS_F16, F32: pvs.PVS_F32}[dtype]
    return pvs.pvs_xent_args(p, p, p, None, rows, items, dim, dim, -100, dim, code, 1.0, 0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V", [(1 << 20, 1 << 20), (1 << 24, 100_000), (5000, 100_000_000)])
def test_loss_scratch_is_bounded(T, V, dtype):
    # statistics of a block of rows, and copies of a piece of the items
    size = ctypes.c_size_t()
    a = xent_args(T, V, 64, dtype)
    assert pvs._lib.pvs_xent_workspace(ctypes.byref(a), 0, ctypes.byref(size)) == pvs.PVS_OK
    assert size.value <= max(2 * GB, 32 * V + GB)


@pytest.mark.parametrize("dtype,T,V", [(BF16, 200_003, 200_000), (F32, 180_000, 200_000), (F32, 171_530, 200_000)])
def test_loss_in_blocks_of_rows(dtype, T, V):
    # more than 1 GB of statistics; the last block of one call has a few rows
    d, scale = 8, 3.0
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(T, d, generator=g, device="cuda").to(dtype)
    w = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    loss, stats = pvs.pvs_xent_forward(x, w, y, scale=scale)
    assert torch.isfinite(loss).all() and torch.isfinite(stats).all()
    for at in (slice(0, 40), slice(171_500, 171_530), slice(T - 40, T)):
        l = scale * (x[at].double() @ w.double().T)
        want = torch.logsumexp(l, dim=1) - l.gather(1, y[at][:, None])[:, 0]
        e = (d / 16 + 4) * 2.0 ** -23 * scale * (x[at].double().abs() @ w.double().abs().T).amax(dim=1)
        close(loss[at], want, 2 * e + 2.0 ** -21 * l.abs().amax(dim=1) + 2.0 ** -19)
        # s 2^m is the sum of the exponentials
        total = torch.log(stats[at, 1].double()) + stats[at, 0].double() * 0.6931471805599453
        close(total, torch.logsumexp(l, dim=1), 2 * e + 2.0 ** -21 * l.abs().amax(dim=1) + 2.0 ** -19)


@pytest.mark.parametrize("T,V", [(1, 500_000_000), (16, 100_000_000), (9, 2_000_000_000)])
def test_gradient_scratch_of_few_rows_is_bounded(T, V):
    size = ctypes.c_size_t()
    a = xent_args(T, V, 64, F32)
    assert pvs._lib.pvs_xent_workspace(ctypes.byref(a), 1, ctypes.byref(size)) == pvs.PVS_OK
    assert size.value <= GB + GB // 4


@pytest.mark.parametrize("T,V", [(5, 40_000_003), (12, 17_000_000)])
def test_gradients_of_few_rows_in_pieces_of_the_items(T, V):
    # more than 1 GB of G, for 8 and for 16 rows; a target and a share of every softmax in
    # each piece, masked items too.  A thread adds about V / 2,400 items, 200 sums join them.
    d, scale = 4, 2.0
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(T, d, generator=g, device="cuda")
    w = torch.rand(V, d, generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[0], y[1], y[2] = 0, V - 1, -100
    bias = torch.randn(V, generator=g, device="cuda")
    bias[::7] = -torch.inf
    bias[y[y >= 0]] = 1.0
    grad = torch.rand(T, generator=g, device="cuda") + 0.5
    _, stats = pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
    dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, bias=bias, scale=scale)
    W = w.double()
    for t in range(T):
        X = x[t].double()
        l = scale * (W @ X) + bias.double()
        G = torch.softmax(l, dim=0)
        if t != 2:
            G[y[t]] -= 1.0
        G *= float(grad[t]) if t != 2 else 0.0
        e = float(((d / 16 + 4) * 2.0 ** -23 * scale * (W @ X.abs())).max()) + 2.0 ** -22 * 30
        rel = 2 * e + 2.0 ** -19 + (V / 2400 + 200) * 2.0 ** -23
        close(dx[t], scale * (G @ W), rel * scale * (G.abs() @ W) + 2.0 ** -126)
        if t == 0:
            want, tol = torch.zeros_like(W), torch.zeros_like(W)
        want += scale * G[:, None] * X
        tol += scale * (2 * e + 2.0 ** -18) * G.abs()[:, None] * X.abs()
    close(dw, want, tol + 2.0 ** -126)
