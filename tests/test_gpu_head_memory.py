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
