"""What the head's operators lose beside the rounding of their outputs.

Bounds taken before any run.  16-bit gradients: G and kept rows enter their products in two
16-bit parts, cut to the first and rounded to the second, which leaves 2^-15 of an
entry (f16 less); a logit's error e is that of the other tests; each of the two
products has its steps of 2^-23.  GELU in float32: x / sqrt(2) is off by 2^-23 of itself, which
moves 1 - Phi by x^2 + 1 times that, erfcf by four last bits, a product by a half; the
exponential's argument by x^2 / 4 times 2^-23, itself and its factors by four last bits.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_ckpt import rows  # noqa: E402
from test_gpu_head_xent import BF16, F16, F32, TINY, UNIT, close, make, reference, step  # noqa: E402

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


@pytest.mark.parametrize("K", [1, 33, 64, 1001, 2100])
def test_float32_gelu_keeps_its_digits(K):
    x = torch.linspace(-13.0, 13.0, 5 * K, device="cuda").reshape(5, K)
    codes, scales, y = pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU)
    X = x.double()
    want = 0.5 * X * torch.erfc(-X / math.sqrt(2.0))
    close(y, want, (X * X + 6) * 2.0 ** -23 * want.abs() + TINY[F32])
    # the slope at what the codes stand for
    X = (codes.float() * scales[:, None]).double()
    dy = torch.linspace(1.0, 2.0, K, device="cuda").expand(5, K).contiguous()
    dx = pvs.pvs_ckpt_act_backward(dy, codes, scales, pvs.PVS_ACT_GELU)
    below = 0.5 * torch.erfc(-X / math.sqrt(2.0))
    beside = X * torch.exp(-0.5 * X * X) / math.sqrt(2.0 * math.pi)
    close(dx, dy.double() * (below + beside),
          (X * X + 8) * 2.0 ** -23 * (below + beside.abs()) * dy.double() + TINY[F32])


# float32 sums of terms of one sign.  Each step of 16 in the tensor cores cuts the running sum,
# by half of 2^-23 of it on average at most, and a split's running sum is half of its last
# one on average: n steps cost n / 2 times 2^-24 in the mean over many entries.  Four more for
# the logits, the operands' parts and the sums of the splits, which round.
def mean_error(got, want):
    return float(((got.double() - want).abs() / want).mean())


@pytest.mark.parametrize("R,N,K", [(25_103, 1093, 122), (24_983, 893, 1860), (4096, 2048, 2048)])
def test_float32_weight_gradients_of_many_rows(R, N, K):
    codes, scales, _ = pvs.pvs_ckpt_store(rows(R, K, F32, 4, spread=0.5).abs())
    dy = rows(R, N, F32, 5, spread=0.5).abs()
    dw = pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    want = dy.double().T @ (codes.double() * scales.double()[:, None])
    assert mean_error(dw, want) <= (64 / 2 + 4) * 2.0 ** -24


@pytest.mark.parametrize("T,V,d", [(6320, 3384, 128), (2000, 2000, 1024), (777, 20_011, 385)])
def test_float32_gradients_of_many_rows(T, V, d):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.rand(T, d, generator=g, device="cuda") / d ** 0.5
    w = torch.rand(V, d, generator=g, device="cuda")
    grad = torch.rand(T, generator=g, device="cuda") + 0.5
    # the target is masked: it has no gradient, and every entry of G is positive
    bias = torch.zeros(V, device="cuda")
    bias[0] = -torch.inf
    y = torch.zeros(T, dtype=torch.int64, device="cuda")
    _, stats = pvs.pvs_xent_forward(x, w, y, bias=bias)
    dx, dw = pvs.pvs_xent_backward(x, w, y, stats, grad, bias=bias)
    G = torch.softmax(x.double() @ w.double().T + bias.double(), dim=1) * grad.double()[:, None]
    assert mean_error(dx, G @ w.double()) <= (32 / 2 + 4) * 2.0 ** -24
    assert mean_error(dw[1:], (G.T @ x.double())[1:]) <= (32 / 2 + 4) * 2.0 ** -24
