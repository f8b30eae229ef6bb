"""Device-side waits of the head's products that run out: the kernel returns, the next call
says so once, and calls after it are right.  A limit of 0 makes a wait give up unless
what it waits for is there already: nothing is made to hang or to fault."""
import time

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

from test_gpu_head_ckpt import rows  # noqa: E402
from test_gpu_head_xent import BF16, F16, F32, make  # noqa: E402

pytestmark = pytest.mark.gpu

LIMIT = 2_000_000_000


def run_out(call):
    """The call under a limit of 0, complete on the device when this returns."""
    pvs.pvs_head_set_wait_limit(0)
    try:
        call()
    finally:
        pvs.pvs_head_set_wait_limit(LIMIT)
    start = time.monotonic()
    torch.cuda.synchronize()
    assert time.monotonic() - start < 1.0


def raised(call):
    with pytest.raises(pvs.PvsError) as e:
        call()
    return e.value.status


# lone CTAs and pairs; one chunk and more chunks than stages; one tile and many; parts
SHAPES = [(100, 5000, 768), (100, 40, 16), (300, 5000, 768), (300, 40, 16), (1000, 20_011, 385)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,d", SHAPES)
def test_cross_entropy(T, V, d, dtype):
    x, w, y, bias, grad, scale = make(T, V, d, dtype, masked=0.1)

    def forward():
        return pvs.pvs_xent_forward(x, w, y, bias=bias, scale=scale)
    loss, stats = forward()

    def backward():
        return pvs.pvs_xent_backward(x, w, y, stats, grad, bias=bias, scale=scale)
    dx, dw = backward()
    for _ in range(10):
        for call, want in ((forward, (loss, stats)), (backward, (dx, dw))):
            run_out(call)
            assert raised(pvs.pvs_head_status) == pvs.PVS_ERR_TIMEOUT
            assert pvs.pvs_head_status() == pvs.PVS_OK
            for a, b in zip(call(), want):
                assert torch.equal(a, b)
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,N,K", [(64, 100, 40), (5000, 128, 300), (5000, 700, 1000)])
def test_weight_gradient(R, N, K, dtype):
    dy = rows(R, N, dtype, 2)
    codes, scales, _ = pvs.pvs_ckpt_store(rows(R, K, dtype, 1))

    def call():
        return pvs.pvs_ckpt_grad_weight(dy, codes, scales)
    want = call()
    for _ in range(10):
        run_out(call)
        # the next call of its kind says so, and queues nothing
        assert raised(call) == pvs.PVS_ERR_TIMEOUT
        assert torch.equal(call(), want)


def test_limits():
    assert raised(lambda: pvs.pvs_head_set_wait_limit(-1)) == pvs.PVS_ERR_INVALID
    # at the limit's maximum and above it, ordinary calls do not run out
    x, w, y, _, _, scale = make(300, 5000, 64, BF16)
    want = pvs.pvs_xent_forward(x, w, y, scale=scale)[0]
    for ns in (1 << 62, LIMIT):
        pvs.pvs_head_set_wait_limit(ns)
        assert torch.equal(pvs.pvs_xent_forward(x, w, y, scale=scale)[0], want)
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK


def entry_points():
    x, w, y, _, grad, scale = make(200, 900, 64, BF16)
    _, stats = pvs.pvs_xent_forward(x, w, y, scale=scale)
    codes, scales, _ = pvs.pvs_ckpt_store(x)
    packed, units = pvs.pvs_wq_pack(w, 64)
    return {
        "xent_forward": lambda: pvs.pvs_xent_forward(x, w, y, scale=scale),
        "xent_backward": lambda: pvs.pvs_xent_backward(x, w, y, stats, grad, scale=scale),
        "ckpt_store": lambda: pvs.pvs_ckpt_store(x, act=pvs.PVS_ACT_GELU),
        "ckpt_load": lambda: (pvs.pvs_ckpt_load(codes, scales, BF16),),
        "ckpt_act_backward": lambda: (pvs.pvs_ckpt_act_backward(x, codes, scales),),
        "ckpt_grad_weight": lambda: (pvs.pvs_ckpt_grad_weight(x, codes, scales),),
        "wq_pack": lambda: pvs.pvs_wq_pack(w, 64),
        "wq_unpack": lambda: (pvs.pvs_wq_unpack(packed, units, 64, 64, BF16),),
        "wq_matvec": lambda: (pvs.pvs_wq_matvec(x[:3], packed, units, 64),),
    }


@pytest.mark.parametrize("name", ["xent_forward", "xent_backward", "ckpt_store", "ckpt_load", "ckpt_act_backward",
                                  "ckpt_grad_weight", "wq_pack", "wq_unpack", "wq_matvec"])
def test_the_next_call_of_any_kind_reports_it(name):
    calls = entry_points()
    want = calls[name]()
    run_out(calls["xent_forward"])
    assert raised(calls[name]) == pvs.PVS_ERR_TIMEOUT
    assert pvs.pvs_head_status() == pvs.PVS_OK
    for a, b in zip(calls[name](), want):
        assert torch.equal(a, b)
