"""Infinities and NaN where the head's operators have to keep them out, or let them through."""
import math

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_xent import BF16, F16, F32, INF, make, step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T", [1, 5, 150])
@pytest.mark.parametrize("features", [-1.0, 1.0])
@pytest.mark.parametrize("value", [-INF, INF, math.nan])
def test_one_masked_entry_whatever_its_products_sign(T, features, value, dtype):
    # features of one sign (as after a ReLU): an infinity in a masked item gives products
    # of one sign with every row
    x, w, y, _, grad, scale = make(T, 300, 64, dtype)
    x = features * x.abs()
    bias = torch.zeros(300, device="cuda")
    y = y.clamp(max=298)
    bias[299] = -INF
    w[299] = 0.5
    clean = step(x, w, y, bias, grad, scale)
    w[299, 17] = value
    for a, b in zip(step(x, w, y, bias, grad, scale), clean):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("K", [1, 33, 64, 1001, 2100])
def test_gelu_of_infinities(K, dtype):
    # x Phi(x): +inf at +inf, NaN at -inf (-inf times 0) and at NaN
    x = torch.linspace(-4.0, 4.0, 3 * K, device="cuda").reshape(3, K).to(dtype)
    want = torch.nn.functional.gelu(x.double())
    x[0, K // 2], x[1, K - 1], x[2, 0] = INF, -INF, math.nan
    want[0, K // 2], want[1, K - 1], want[2, 0] = INF, math.nan, math.nan
    codes, scales, y = pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU)
    assert torch.isnan(scales).all() and not codes.any()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y == INF, want == INF)
    fine = torch.isfinite(want)
    assert torch.allclose(y.double()[fine], want[fine], rtol=2.0 ** -7, atol=2.0 ** -18)
