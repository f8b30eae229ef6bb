"""Softmax cross entropy over a large vocabulary and its gradients against the
definition in binary64.

Tolerances are bounds on the rounding of the kernels, taken before any run:
a logit of d products summed in float32 steps of 16 is off by at most
e = (d / 16 + 4) 2^-23 a sum|x w| + 2^-22 |l| (sums may be cut, not rounded); a
loss by 2 e + 2^-19 (the exponentials' and the sum's own error) and 2^-22 of
itself; an entry of G by its type's rounding and 2 e + 2^-19 of itself; a
gradient by that through sum|G w|, its own steps, and its type's rounding.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 2.0 ** -126, F16: 2.0 ** -24, F32: 2.0 ** -126}
INF = math.inf


def make(T, V, d, dtype, seed=0, masked=0.0, ignored=0.0, spread=4.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(T, d, generator=g, device="cuda") / d ** 0.5).to(dtype)
    w = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    bias = None
    if masked:
        bias = torch.randn(V, generator=g, device="cuda")
        bias[torch.rand(V, generator=g, device="cuda") < masked] = -INF
        bias[y] = 0.25
    if ignored:
        y[torch.rand(T, generator=g, device="cuda") < ignored] = -100
    grad = torch.randn(T, generator=g, device="cuda") / T
    return x, w, y, bias, grad, spread


def reference(x, w, y, bias, grad, scale):
    """loss, dx, dw of the definition in binary64, and their tolerances."""
    X, W = x.double(), w.double()
    d = X.shape[1]
    out = torch.zeros(W.shape[0], dtype=torch.bool, device=x.device)
    if bias is not None:
        out = bias == -INF
    W0 = torch.where(out[:, None], torch.zeros_like(W), W)
    kept = y != -100
    X0 = torch.where(kept[:, None], X, torch.zeros_like(X))
    l = scale * (X0 @ W0.T)
    if bias is not None:
        l = l + bias.double()
    at = y.clamp(min=0)[:, None]
    none = (out.all() | ~kept)
    lse = torch.logsumexp(l, dim=1)
    loss = torch.where(none, torch.zeros_like(lse), lse - l.gather(1, at)[:, 0])
    p = torch.exp(l - lse[:, None])
    p = torch.where(none[:, None], torch.zeros_like(p), p)
    G = p.clone()
    # p - 1 of the target as the others' negative sum: p near 1 loses no digits
    visible = ~none & ~out[at[:, 0]]
    G.scatter_(1, at, 0.0)
    G.scatter_(1, at, torch.where(visible, -G.sum(dim=1), torch.zeros_like(lse))[:, None])
    G = G * grad.double()[:, None]
    size = scale * (X0.abs() @ W0.abs().T)
    lf = torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
    e = ((d / 16 + 4) * 2.0 ** -23 * size + 2.0 ** -22 * lf).amax(dim=1)
    tol_loss = 2 * e + 2.0 ** -19 + 2.0 ** -22 * loss.abs()
    unit = UNIT[x.dtype]
    g_rel = unit + 2 * e + 2.0 ** -19
    A = G.abs() * g_rel[:, None]
    if x.dtype == F16:   # entries below the scaled f16's last bit
        A = A + grad[kept].abs().max().double() * 2.0 ** -37 if kept.any() else A
    aG = G.abs()
    dx, dw = scale * (G @ W0), scale * (G.T @ X0)
    tdx = scale * (A @ W0.abs()) + (W.shape[0] / 16 + 8) * 2.0 ** -23 * scale * (aG @ W0.abs())
    tdw = scale * (A.T @ X0.abs()) + (X.shape[0] / 16 + 8) * 2.0 ** -23 * scale * (aG.T @ X0.abs())
    tdx = tdx + unit * dx.abs() + TINY[x.dtype]
    tdw = tdw + unit * dw.abs() + TINY[x.dtype]
    return (loss, dx, dw), (tol_loss, tdx, tdw)


def close(got, want, tol):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got - want).abs()[fine]
    over = off > tol.expand_as(want)[fine]
    assert not over.any(), (float(off[over].max()), int(over.sum()), off.numel())


def step(x, w, y, bias, grad, scale, **kw):
    loss, stats = pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
    dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, bias=bias, scale=scale, **kw)
    return loss, dx, dw


def check(case):
    got = step(*case)
    want, tol = reference(*case)
    for a, b, t in zip(got, want, tol):
        assert a.dtype in (case[0].dtype, F32)
        close(a, b, t)
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK
    return got


SHAPES = [(1, 1, 1), (1, 2, 3), (2, 17, 8), (1, 10_000, 128), (127, 255, 64), (128, 256, 256),
          (129, 257, 65), (300, 1000, 385), (33, 4097, 768), (1000, 100, 1024), (5, 70_001, 24),
          (4096, 300, 40), (257, 999, 513), (16, 513, 2000)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,d", SHAPES)
def test_step_matches_definition(T, V, d, dtype):
    check(make(T, V, d, dtype))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,d", [(1, 300, 16), (200, 777, 136), (130, 3000, 385)])
@pytest.mark.parametrize("masked,ignored", [(0.5, 0.0), (0.02, 0.3), (0.97, 0.9)])
def test_masks_and_ignored_rows(T, V, d, dtype, masked, ignored):
    check(make(T, V, d, dtype, masked=masked, ignored=ignored))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_several_pieces_of_the_vocabulary(dtype):
    # the gradient of every logit would be 0.5 to 1.6 GB here: several pieces
    check(make(8192, 33_001, 24, dtype, masked=0.1, ignored=0.1))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_strided_and_unaligned_operands(dtype):
    x, w, y, bias, grad, scale = make(70, 501, 96, dtype)
    for d, off in ((96, 0), (90, 3), (33, 1)):
        xs = torch.full((70, 140), float("nan"), dtype=dtype, device="cuda")
        ws = torch.full((501, 123), float("nan"), dtype=dtype, device="cuda")
        xs[:, off:off + d] = x[:, :d]
        ws[:, off:off + d] = w[:, :d]
        check((xs[:, off:off + d], ws[:, off:off + d], y, None, grad, scale))
    # columns first, every other row, and one row for all
    check((x.T.contiguous().T, w.T.contiguous().T, y, None, grad, scale))
    check((x[::2], w[::3], y[::2] % 167, None, grad[::2], scale))
    check((x[:1].expand(70, 96), w, y, None, grad, scale))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_nothing_in_the_softmax(dtype):
    x, w, y, _, grad, scale = make(40, 300, 64, dtype)
    bias = torch.full((300,), -INF, device="cuda")
    loss, dx, dw = step(x, w, y, bias, grad, scale)
    assert not loss.any() and not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_masked_items_and_ignored_rows_may_hold_anything(dtype):
    x, w, y, bias, grad, scale = make(150, 900, 72, dtype, masked=0.2, ignored=0.2)
    clean = step(x, w, y, bias, grad, scale)
    w2, x2 = w.clone(), x.clone()
    out = torch.nonzero(bias == -INF)[:, 0]
    w2[out[::3]] = float("nan")
    w2[out[1::3]] = INF
    w2[out[2::3], 5] = -INF
    x2[y == -100] = float("nan")
    x2[torch.nonzero(y == -100)[0, 0], 3] = INF
    for a, b in zip(step(x2, w2, y, bias, grad, scale), clean):
        assert torch.equal(a, b)


def test_every_row_ignored():
    x, w, _, _, grad, scale = make(64, 200, 32, BF16)
    y = torch.full((64,), -100, device="cuda")
    for out in step(x, w, y, None, grad, scale):
        assert not out.any()
    loss, stats = pvs.pvs_xent_forward(x, w, torch.full_like(y, 7), ignore_index=7)
    assert not loss.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_lowest_value_biases(dtype):
    # finite biases of the type's lowest value are not -inf: among themselves they
    # are alike, next to others they do not count
    x, w, y, _, grad, scale = make(9, 64, 32, dtype)
    low = torch.finfo(F32).min
    bias = torch.full((64,), low, device="cuda")
    loss, stats = pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
    assert torch.allclose(loss.double(), torch.full_like(loss, math.log(64)).double(), rtol=2 ** -19)
    bias[:32] = 0.0
    y = torch.arange(9, device="cuda")
    check((x, w, y, torch.where(bias == 0, bias, torch.full_like(bias, low)), grad, scale))
    loss, _ = pvs.pvs_xent_forward(x, w, torch.full_like(y, 50), bias=bias, scale=scale)
    assert torch.allclose(loss.double(), torch.full_like(loss, -low).double(), rtol=2 ** -19)


def test_masked_target_and_target_alone():
    x, w, y, _, grad, scale = make(20, 100, 48, BF16)
    bias = torch.zeros(100, device="cuda")
    bias[y] = -INF
    check((x, w, y, bias, grad, scale))
    # only one item left: certain, no loss and no gradient
    bias = torch.full((100,), -INF, device="cuda")
    bias[7] = 3.0
    loss, dx, dw = step(x, w, torch.full_like(y, 7), bias, grad, scale)
    assert not loss.any() and not dx.any() and not dw.any()


def test_targets_out_of_range_and_non_finite_rows():
    x, w, y, _, grad, scale = make(6, 50, 16, F32)
    y = torch.tensor([3, 50, -1, 4, 2 ** 40, 5], device="cuda")
    loss, dx, dw = step(x, w, y, None, grad, scale)
    bad = torch.tensor([False, True, True, False, True, False], device="cuda")
    assert torch.equal(torch.isnan(loss), bad)
    assert torch.equal(torch.isnan(dx).all(dim=1), bad) and torch.isnan(dw).all()
    x[2, 3] = float("nan")
    loss, _ = pvs.pvs_xent_forward(x, w, torch.arange(6, device="cuda"), scale=scale)
    assert torch.equal(torch.isnan(loss), torch.arange(6, device="cuda") == 2)


def test_large_logits_and_certain_rows():
    # logits of hundreds; losses of 1e-8 and of hundreds keep their digits
    x, w, y, _, grad, _ = make(64, 300, 64, F32)
    w[y] = 3.0 * x / x.norm(dim=1, keepdim=True) * 8.0
    check((x, w, y, None, grad, 3.0))
    check((x, w, (y + 1) % 300, None, grad, 40.0))


def test_gradient_against_differences():
    # central differences of the summed loss along a direction: the float32 loss is
    # off by tol a row, and the third derivative of a log-sum-exp along a
    # direction with |dl| <= r is at most 2 r^3
    x, w, y, bias, grad, scale = make(24, 130, 40, F32, masked=0.1, spread=1.0)
    grad = grad.abs() + 0.01
    _, (tol, _, _) = reference(x, w, y, bias, grad, scale)
    _, stats = pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
    dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, bias=bias, scale=scale)
    g = torch.Generator(device="cuda").manual_seed(5)
    h = 2.0 ** -6

    def total(x, w):
        loss, _ = pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
        return (loss.double() * grad.double()).sum()
    for which in (0, 1):
        v = torch.randn(*(x, w)[which].shape, generator=g, device="cuda")
        v = v / (1.0 if which == 0 else 40 ** 0.5)
        plus = (x + h * v, w) if which == 0 else (x, w + h * v)
        minus = (x - h * v, w) if which == 0 else (x, w - h * v)
        slope = (total(*plus) - total(*minus)) / (2 * h)
        r = scale * (v @ w.T if which == 0 else x @ v.T).abs().amax(dim=1).double()
        err = ((grad.double() * (tol / h + 2 * r ** 3 * h * h / 6 * 2)).sum()
               + 2.0 ** -20 * ((dx, dw)[which].double() * v.double()).abs().sum())
        assert abs(slope - ((dx, dw)[which].double() * v.double()).sum()) <= err


def test_one_gradient_alone_and_repeatable():
    case = make(500, 3000, 200, BF16, masked=0.05, ignored=0.1)
    x, w, y, bias, grad, scale = case
    loss, dx, dw = step(*case)
    loss2, dx2, none = step(*case, need_w=False)
    assert none is None and torch.equal(loss, loss2) and torch.equal(dx, dx2)
    _, none, dw2 = step(*case, need_x=False)
    assert none is None and torch.equal(dw, dw2)
    assert step(*case, need_x=False, need_w=False)[1:] == (None, None)


def test_f16_gradients_of_scaled_losses():
    for up in (2.0 ** -30, 1.0, 65536.0, 2.0 ** 100):
        x, w, y, _, grad, scale = make(64, 500, 64, F16)
        grad = grad * up
        loss, stats = pvs.pvs_xent_forward(x, w, y, scale=scale)
        dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, scale=scale)
        want, tol = reference(x, w, y, None, grad, scale)
        for a, b, t in ((dx, want[1], tol[1]), (dw, want[2], tol[2])):
            fits = b.abs() + t < 65504.0
            close(torch.where(fits, a.double(), b), b, t)


def test_other_streams_and_graphs():
    case = make(200, 2000, 128, BF16, ignored=0.1)
    want = step(*case)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(*case)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*case)
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_offsets_past_32_bits():
    # 2.4e9 elements of w: the last items are reached, and their gradient written
    T, V, d = 3, 3_100_000, 768
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(V, d, dtype=BF16, device="cuda")
    for i in range(0, V, 1 << 18):
        n = min(1 << 18, V - i)
        w[i:i + n] = torch.randn(n, d, generator=g, device="cuda") / d ** 0.5
    y = torch.tensor([V - 1, 5, V - 200_000], device="cuda")
    x = w[y].clone()
    scale = 12.0
    grad = torch.ones(T, device="cuda")
    loss, stats = pvs.pvs_xent_forward(x, w, y, scale=scale)
    dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, scale=scale)
    l = torch.cat([scale * (x.double() @ w[i:i + (1 << 18)].double().T)
                   for i in range(0, V, 1 << 18)], dim=1)
    lse = torch.logsumexp(l, dim=1)
    assert torch.allclose(loss.double(), lse - l.gather(1, y[:, None])[:, 0], rtol=0, atol=1e-4)
    tail = slice(V - 250_000, V)
    G = torch.exp(l - lse[:, None])
    G[torch.arange(T, device="cuda"), y] -= 1.0
    want = scale * (G[:, tail].T @ x.double())
    size = scale * (G[:, tail].abs().T @ x.double().abs())
    close(dw[tail], want, 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1e-4) * size + 2.0 ** -126)


def test_no_rows():
    x, w, y, _, grad, _ = make(4, 50, 16, BF16)
    loss, dx, dw = step(x[:0], w, y[:0], None, grad[:0], 1.0)
    assert loss.shape == (0,) and dx.shape == (0, 16) and dw.shape == (50, 16) and not dw.any()


def test_refusals():
    x, w, y, _, grad, scale = make(8, 60, 32, BF16)
    bias = torch.zeros(60, device="cuda")
    f = pvs.pvs_xent_forward
    for exc, args, kw in [
            (TypeError, (x.cpu(), w, y), {}), (TypeError, (x, w.float(), y), {}),
            (TypeError, (x.double(), w.double(), y), {}), (TypeError, (x, w, y.int()), {}),
            (TypeError, (x, w, y), dict(bias=bias.half())),
            (ValueError, (x, w[:, :16], y), {}), (ValueError, (x, w, y[:4]), {}),
            (ValueError, (x[0], w, y), {}), (ValueError, (x, w[:0], y), {}),
            (ValueError, (x, w, y), dict(bias=bias[:7])), (ValueError, (x, w, y), dict(scale=0.0)),
            (ValueError, (x, w, y), dict(scale=float("inf"))),
            (ValueError, (x[:, :0], w[:, :0], y), {})]:
        with pytest.raises(exc):
            f(*args, **kw)
    _, stats = f(x, w, y)
    with pytest.raises(ValueError):
        pvs.pvs_xent_backward(x, w, y, stats[:4], grad)
    with pytest.raises(ValueError):
        pvs.pvs_xent_backward(x, w, y, stats, grad[:4])
    with pytest.raises(TypeError):
        pvs.pvs_xent_backward(x, w, y, stats, grad.half())


def test_float32_rows_and_items_of_unlike_sizes():
    # rows and items from 2^-60 to 2^60 of one another: each logit and gradient keeps the
    # digits that its own products have
    x, w, y, _, grad, scale = make(40, 300, 72, F32, spread=1.0)
    up = torch.exp2(torch.randint(-60, 61, (40, 1), device="cuda").float())
    down = torch.exp2(torch.randint(-60, 61, (300, 1), device="cuda").float())
    check((x * up, w / up.max(), y, None, grad, scale))
    check((x / down.max(), w * down, y, None, grad, scale))
    # the largest and the smallest that float32 holds, with logits of order one
    check((x * 2.0 ** 120, w * 2.0 ** -120, y, None, grad, scale))
    check((x * 2.0 ** -100, w * 2.0 ** 100, y, None, grad, scale))
