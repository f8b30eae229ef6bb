"""f16 gradients of losses times a power of two: what f16 holds, with the right sign; what
it cannot, as infinities of that sign."""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_xent import F16, INF, TINY, close, make, reference, step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [12, 64, 300])
@pytest.mark.parametrize("up", [-16, -10, 0, 12])
def test_gradients_that_f16_holds(up, T):
    x, w, y, _, grad, scale = make(T, 500, 64, F16)
    grad = grad * 2.0 ** up
    _, dx, dw = step(x, w, y, None, grad, scale)
    (_, want_x, want_w), (_, tol_x, tol_w) = reference(x, w, y, None, grad, scale)
    # (the bounds of the other tests, with half of f16's last bit for its rounding)
    close(dx, want_x, tol_x - TINY[F16] / 2)
    close(dw, want_w, tol_w - TINY[F16] / 2)
    if up >= -10:
        # (about the wanted values alone: a zero or a wrong sign fails at most of them)
        assert (want_x.abs() > tol_x).float().mean() > 0.5


@pytest.mark.parametrize("T", [12, 64, 300])
@pytest.mark.parametrize("up", [40, 100])
def test_gradients_beyond_f16(up, T):
    x, w, y, _, grad, scale = make(T, 500, 64, F16)
    grad = grad * 2.0 ** up
    _, dx, dw = step(x, w, y, None, grad, scale)
    (_, want_x, want_w), (_, tol_x, tol_w) = reference(x, w, y, None, grad, scale)
    for got, want, tol in ((dx, want_x, tol_x), (dw, want_w, tol_w)):
        beyond = want.abs() - tol > 65520.0
        assert beyond.float().mean() > 0.5
        assert torch.equal(got[beyond].double(), torch.sign(want[beyond]) * INF)
        assert not torch.isnan(got).any()
