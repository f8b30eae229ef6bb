"""Distillation of rows whose logits are all -inf: the formula has no value there, and every output
that such a row reaches says so, as it does for a row of NaN.  Rows without a list stay without a
loss, and the other rows as they are without the bad ones."""
import math

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = math.inf


def step(x, w, ids, z, grad, bias):
    loss, stats, hits = pvs.pvs_distill_forward(x, w, ids, z, bias=bias)
    dx, dw = pvs.pvs_distill_backward(x, w, ids, stats, hits, grad, bias=bias)
    return loss, dx, dw


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,K", [(5, 4, 4), (5, 300, 7), (50, 4, 4), (50, 300, 7), (700, 1000, 20)])
def test_every_logit_minus_infinite(T, V, K, dtype, masked):
    d = 64
    g = torch.Generator(device="cuda").manual_seed(7)
    w = (torch.rand(V, d, generator=g, device="cuda") + 0.5).to(dtype)
    x = (torch.randn(T, d, generator=g, device="cuda") / 8.0).to(dtype)
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(T)])
    z = torch.randn(T, K, generator=g, device="cuda")
    grad = torch.rand(T, generator=g, device="cuda") + 0.5
    bias = None
    if masked:
        bias = torch.zeros(V, device="cuda")
        bias[1] = -INF
    ids[3] = -100
    good = step(x, w, ids, z, grad, bias)
    assert all(torch.isfinite(v).all() for v in good)
    x[2, 0] = x[3, 0] = -INF             # w is positive: the logits of rows 2 and 3 are all -inf
    loss, dx, dw = step(x, w, ids, z, grad, bias)
    rest = torch.arange(T, device="cuda") != 2
    assert torch.isnan(loss[2]) and torch.isnan(dx[2]).all()
    assert torch.equal(loss[rest], good[0][rest]) and loss[3] == 0
    assert torch.equal(dx[rest], good[1][rest]) and not dx[3].any()
    kept = torch.ones(V, dtype=torch.bool, device="cuda") if bias is None else bias == 0.0
    assert torch.isnan(dw[kept]).all()
