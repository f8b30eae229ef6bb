"""What the head's operators lose beside the rounding of their outputs.

Bounds taken before any run.  16-bit gradients: G and kept rows enter their products in two
16-bit parts, cut to the first and rounded to the second, which leaves 2^-15 of an
entry (f16 less); a logit's error e is that of the other tests; each of the two
products has its steps of 2^-23.
"""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_ckpt import rows  # noqa: E402
from test_gpu_head_xent import BF16, F16, TINY, UNIT, close, make, reference, step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,V,d", [(129, 40, 16), (300, 64, 24), (1000, 33, 8), (2000, 700, 40)])
def test_16_bit_gradients_of_many_rows(T, V, d, dtype):
    x, w, y, bias, grad, scale = make(T, V, d, dtype, masked=0.1)
    _, dx, dw = step(x, w, y, bias, grad, scale)
    (_, want_x, want_w), _ = reference(x, w, y, bias, grad, scale)
    X, W = x.double(), torch.where((bias == -torch.inf)[:, None], 0.0, w.double())
    l = scale * (X @ W.T) + bias.double()
    G = (torch.softmax(l, dim=1) - torch.nn.functional.one_hot(y, V)) * grad.double()[:, None]
    finite = torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
    e = ((d / 16 + 4) * 2.0 ** -23 * scale * (X.abs() @ W.abs().T) + 2.0 ** -22 * finite).amax(dim=1)
    aG = G.abs() * (2.0 ** -15 + 2 * e + 2.0 ** -19)[:, None]
    if dtype == F16:   # entries below the scaled f16's last bit
        aG = aG + grad.abs().max().double() * 2.0 ** -37
    unit = UNIT[dtype] * 1.001
    for got, want, a, g, other in ((dx, want_x, aG, G.abs(), W.abs()),
                                   (dw, want_w, aG.T, G.abs().T, X.abs())):
        steps = 2 * (other.shape[0] / 16 + 8) * 2.0 ** -23
        close(got, want, scale * (a @ other + steps * (g @ other)) + unit * want.abs() + TINY[dtype])


@pytest.mark.parametrize("R,N,K", [(7, 9, 17), (64, 128, 256), (300, 130, 385), (1000, 72, 40)])
def test_bf16_weight_gradients(R, N, K):
    x, dy = rows(R, K, BF16, 4, spread=0.5), rows(R, N, BF16, 5, spread=0.5)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    kept = codes.double() * scales.double()[:, None]
    want = dy.double().T @ kept
    size = dy.double().abs().T @ kept.abs()
    close(dw, want, (2.0 ** -15 + 2 * (R / 16 + 8) * 2.0 ** -23) * size
          + UNIT[BF16] * 1.001 * want.abs() + TINY[BF16])
