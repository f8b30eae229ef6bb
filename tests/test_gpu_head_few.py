"""Softmax cross entropy of few rows: up to 16 float32 rows, which take the items as they
lie, and up to 128 of 16 bits, whose gradients are as exact as their own rounding.

Against the same definition in binary64 and with the same bounds as the other row
counts: a logit's float32 sum has d / 32 + 5 steps here, a sum over items one step for
each of a thread's items, of a block's groups and of the blocks, all fewer than the
steps that those bounds allow.
"""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_xent import (BF16, F16, F32, INF, TINY, UNIT, check, close, make,  # noqa: E402
                                reference, step)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 7, 8, 9, 16, 17])
@pytest.mark.parametrize("V,d", [(1, 5), (31, 64), (33, 65), (300, 1), (1000, 1024), (1000, 1025),
                                 (5003, 385), (20_011, 768), (70_001, 100)])
def test_step_matches_definition(T, V, d):
    check(make(T, V, d, F32, seed=T))


@pytest.mark.parametrize("T,V,d", [(1, 300, 16), (8, 4001, 384), (16, 777, 130)])
@pytest.mark.parametrize("masked,ignored", [(0.5, 0.0), (0.02, 0.3), (0.97, 0.9)])
def test_masks_and_ignored_rows_hold_anything(T, V, d, masked, ignored):
    x, w, y, bias, grad, scale = make(T, V, d, F32, masked=masked, ignored=ignored)
    w[bias == -INF] = float("nan")
    x[y == -100] = INF
    check((x, w, y, bias, grad, scale))


@pytest.mark.parametrize("d,off", [(96, 0), (90, 3), (33, 1), (64, 2)])
def test_strided_and_unaligned_operands(d, off):
    x, w, y, bias, grad, scale = make(11, 501, 96, F32, masked=0.1)
    xs = torch.full((11, 140), float("nan"), device="cuda")
    ws = torch.full((501, 137), float("nan"), device="cuda")
    xs[:, off:off + d] = x[:, :d]
    ws[:, off:off + d] = w[:, :d]
    check((xs[:, off:off + d], ws[:, off:off + d], y, bias, grad, scale))


def test_one_gradient_alone_and_repeatable():
    case = make(13, 9001, 200, F32, masked=0.05, ignored=0.2)
    loss, dx, dw = check(case)
    for want in ({"need_w": False}, {"need_x": False}):
        again = step(*case, **want)
        assert torch.equal(again[0], loss)
        for got, full in ((again[1], dx), (again[2], dw)):
            assert got is None or torch.equal(got, full)


def test_certain_rows_and_large_logits():
    x, w, y, bias, grad, _ = make(6, 900, 48, F32)
    x[:3] = 4 * w[y[:3]]
    check((x, w, y, bias, grad, 30.0))


def test_nothing_in_the_softmax():
    x, w, y, _, grad, scale = make(9, 100, 72, F32)
    bias = torch.full((100,), -INF, device="cuda")
    loss, dx, dw = step(x, w, y, bias, grad, scale)
    for got in (loss, dx, dw):
        assert torch.equal(got, torch.zeros_like(got))


def test_gradient_against_differences():
    # the loss of 5 rows along a direction: a central difference in binary64's reference
    # bounds the formula, the kernel's gradient is compared with that formula
    case = make(5, 40, 24, F32)
    x, w, y, bias, grad, scale = case
    _, dx, dw = step(*case)
    g = torch.Generator(device="cuda").manual_seed(3)
    u = torch.randn(x.shape, generator=g, device="cuda").double()
    v = torch.randn(w.shape, generator=g, device="cuda").double()

    def total(h):
        l = scale * ((x.double() + h * u) @ (w.double() + h * v).T)
        return ((torch.logsumexp(l, 1) - l.gather(1, y[:, None])[:, 0]) * grad.double()).sum()

    h = 1e-5
    slope = (total(h) - total(-h)) / (2 * h)
    along = (dx.double() * u).sum() + (dw.double() * v).sum()
    _, (_, tdx, tdw) = reference(*case)
    # the difference's own error: h^2 times a third derivative of order (scale |u| |w|)^3, and
    # cancellation of 2^-53 / h
    third = (scale * (u.abs() @ w.double().abs().T + x.double().abs() @ v.abs().T)).amax() ** 3
    tol = (tdx * u.abs()).sum() + (tdw * v.abs()).sum() + h * h * third * grad.abs().sum() + 1e-9
    assert (slope - along).abs() <= tol
    close(dx, reference(*case)[0][1], tdx)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,V,d", [(1, 616, 1024), (10, 866, 200), (128, 3000, 64)])
def test_16_bit_gradients_show_their_own_rounding_only(T, V, d, dtype):
    # G in two parts: cut to 8 bits, the rest rounded to 8 (bf16), 2^-15 of an entry; f16
    # leaves less.  Each of the two products has its steps.  The rest as in the bounds
    # of one part, without that part's rounding.
    x, w, y, bias, grad, scale = make(T, V, d, dtype, masked=0.1)
    _, dx, dw = step(x, w, y, bias, grad, scale)
    (_, want_x, want_w), _ = reference(x, w, y, bias, grad, scale)
    X, W = x.double(), torch.where((bias == -INF)[:, None], 0.0, w.double())
    l = scale * (X @ W.T) + bias.double()
    p = torch.softmax(l, dim=1)
    G = (p - torch.nn.functional.one_hot(y, V)) * grad.double()[:, None]
    finite = torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
    e = ((d / 16 + 4) * 2.0 ** -23 * scale * (X.abs() @ W.abs().T) + 2.0 ** -22 * finite).amax(dim=1)
    aG = G.abs() * (2.0 ** -15 + 2 * e + 2.0 ** -19)[:, None]
    if dtype == F16:   # entries below the scaled f16's last bit
        aG = aG + grad.abs().max().double() * 2.0 ** -37
    unit = UNIT[dtype] * 1.001
    for got, want, other, a, g in ((dx, want_x, W.abs(), aG, G.abs()), (dw, want_w, X.abs(), aG.T, G.abs().T)):
        steps = 2 * (other.shape[0] / 16 + 8) * 2.0 ** -23
        close(got, want, scale * (a @ other + steps * (g @ other)) + unit * want.abs() + TINY[dtype])
