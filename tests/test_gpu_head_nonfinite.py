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
