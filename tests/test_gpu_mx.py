"""Microscaled 4-bit rows and their products against the format's definition in binary64.

Packing is held to the definition to the bit: scales are powers of two, or e4m3 numbers whose
border cases float32 decides exactly, and a code's borders are compared exactly.  A product sums
K exact products of codes and scales in steps of 64 that may be cut, not rounded, to 24 bits of
the largest: (K / 64 + 8) 2^-23 of sum|x w|, its scaling 2^-23 of itself, and half a step of
the output.  Tolerances were taken before any run.
"""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -24, F32: 2.0 ** -149}


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows_of(r, k, dtype, seed=0, spread=1.0):
    g = generator(seed)
    x = torch.randn(r, k, generator=g, device="cuda") * torch.exp(spread * torch.randn(r, 1, generator=g, device="cuda"))
    return (x * torch.exp(spread * torch.randn(1, k, generator=g, device="cuda"))).to(dtype)


def two(e):
    """2^e in binary64 from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def binade(v):
    """floor(log2 v) of positive binary64 numbers (0 for 0)."""
    return torch.frexp(torch.where(v > 0, v, 1.0)).exponent.to(torch.int64) - 1


def nearest(q, low):
    """q to 2 bits behind the leading one's place of e2m1 (1) or e4m3 (3), ties to even."""
    bits = 1 if low == 0 else 3
    step = two(binade(q.abs()).clamp(min=low) - bits)
    return torch.round(q / step) * step


def definition(x, group):
    """Values [R, K], code magnitudes' values [R, padded K] and scales [R, groups] in binary64; NaN
    where the format keeps NaN."""
    r, k = x.shape
    kp = (k + 127) // 128 * 128
    X = torch.zeros(r, kp, dtype=torch.float64, device=x.device)
    X[:, :k] = x.double()
    X = X.view(r, -1, group)
    bad = ~torch.isfinite(X)
    if group == 32:
        bad = bad.any(dim=2, keepdim=True)
        peak = X.abs().amax(dim=2, keepdim=True)
        peak = torch.where(bad, 1.0, peak)
        unit = torch.where(peak > 0, two((binade(peak) - 2).clamp(min=-127)), 2.0 ** -127)
    else:
        bad = bad.any(dim=2, keepdim=True).any(dim=1, keepdim=True)
        peak = torch.where(bad, 0.0, X.abs().amax(dim=2, keepdim=True))
        most = peak.amax(dim=1, keepdim=True)
        row = torch.where(most > 0, two((binade(most) - 10).clamp(min=-126)), 1.0)
        sixth = torch.tensor(1.0 / 6.0, dtype=F32, device=x.device)
        unit = nearest((peak.float() * sixth).double() / row, -6) * row
    q = torch.where(unit > 0, X / torch.where(unit > 0, unit, 1.0), 0.0)
    q = torch.where(bad, 0.0, nearest(q, 0).clamp(-6.0, 6.0))
    unit = torch.where(bad, float("nan"), unit)
    return (q * unit).reshape(r, kp)[:, :k]


def same(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.double()), torch.nan_to_num(want.double()))


def check_pack(x, group):
    codes, scales, rows = pvs.pvs_mx_pack(x, group)
    k = x.shape[1]
    kp = (k + 127) // 128 * 128
    assert codes.shape == (x.shape[0], kp // 2)
    assert scales.shape == ((x.shape[0] + 127) // 128, kp // (4 * group), 512)
    assert (rows is None) == (group == 32)
    got = pvs.pvs_mx_unpack(codes, scales, rows, group, k, F32)
    want = definition(x, group)
    same(got, want.float())
    return codes, scales, rows


PACKED = [(1, 1), (1, 16), (2, 31), (3, 33), (5, 127), (127, 128), (128, 129), (129, 256), (300, 385), (257, 1000),
          (64, 1024), (40, 1025), (33, 2049), (7, 8192), (2, 32_767)]


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("r,k", PACKED)
def test_pack_is_the_definition(r, k, dtype, group):
    check_pack(rows_of(r, k, dtype), group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_borders_between_codes(dtype, group):
    # every border of a code times many scales, and its neighbours in the type
    b = torch.tensor([0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 5.5, 6.0, 7.0], device="cuda")
    s = torch.arange(8, 16, device="cuda", dtype=F32) / 8
    x = (b[None, :] * s[:, None]).to(dtype)
    up = torch.nextafter(x, torch.full_like(x, 100.0))
    dn = torch.nextafter(x, torch.full_like(x, -100.0))
    x = torch.stack((x, up, dn, -x, -up, -dn)).reshape(-1, 16)
    # with and without a largest element that fixes the scale
    y = x.clone()
    y[:, 15] = (6.0 * s).to(dtype).repeat(6)
    z = torch.cat([x, y], dim=1)
    for f in (1.0, 2.0 ** -7, 2.0 ** 9):
        check_pack((z.float() * f).to(dtype), group)
        check_pack((torch.cat([x, y], dim=0).float() * f).to(dtype), group)


@pytest.mark.parametrize("group", [16, 32])
def test_extreme_sizes(group):
    e = torch.arange(-149, 128, device="cuda", dtype=torch.float64)
    x = (two(e)[:, None] * torch.linspace(0.1, 1.99, 64, device="cuda", dtype=torch.float64)[None, :]).clamp(max=3.4e38).float()
    check_pack(x, group)
    check_pack(x.T.contiguous(), group)
    check_pack(torch.zeros(5, 100, device="cuda"), group)
    x = rows_of(9, 300, F32)
    x[1] = 0.0
    x[2, 40:] = 0.0
    x[3, 7] = 3e38
    x[4] *= 1e-38
    check_pack(x, group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_are_not_finite(dtype, group):
    x = rows_of(200, 300, dtype)
    x[3, 5] = float("nan")
    x[130, 299] = float("inf")
    x[131, 128] = -float("inf")
    check_pack(x, group)
    check_pack(x[:, :297], group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_rows(dtype, group):
    x = rows_of(150, 400, dtype)
    for lo, hi in ((0, 384), (1, 258), (3, 400), (8, 72)):
        check_pack(x[:, lo:hi], group)
    check_pack(x[::3], group)
    check_pack(x.T, group)
    check_pack(x[:1].expand(140, 400), group)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_unpack_types(dtype):
    x = rows_of(20, 77, F32, spread=0.3)
    codes, scales, rows = pvs.pvs_mx_pack(x, 16)
    same(pvs.pvs_mx_unpack(codes, scales, rows, 16, 77, dtype), definition(x, 16).to(dtype))


def check_product(x, w, group):
    packed = pvs.pvs_mx_pack(w, group)
    y = pvs.pvs_mx_matmul(x, *packed, group)
    X, W = definition(x, group), definition(w, group)
    want = X @ W.T
    tol = (x.shape[1] / 64 + 8) * 2.0 ** -23 * (X.abs() @ W.abs().T)
    tol = tol + (torch.finfo(x.dtype).eps / 2 + 2.0 ** -23) * want.abs() + TINY[x.dtype]
    assert y.dtype == x.dtype and y.shape == want.shape
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    over = (y.double() - want).abs() > tol
    assert not over.any(), (int(over.sum()), y.numel(), float((y.double() - want).abs()[over].max()))
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK
    return y, packed


PRODUCTS = [(1, 128, 64), (1, 1, 1), (16, 128, 128), (2, 100, 200), (17, 129, 256), (33, 300, 385), (64, 256, 512),
            (100, 1000, 768), (128, 130, 1024), (1, 5000, 771), (3, 64, 8192), (129, 257, 128), (200, 128, 512),
            (256, 256, 256), (257, 700, 333), (300, 40, 4096), (512, 513, 1000), (1000, 2000, 384), (2, 20_000, 4000),
            (1, 128, 32_767), (5000, 3, 64)]


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("b,n,k", PRODUCTS)
def test_product(b, n, k, dtype, group):
    check_product(rows_of(b, k, dtype, 1, 0.3), rows_of(n, k, dtype, 2, 0.3) * k ** -0.5, group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("b", [5, 300])
def test_product_of_any_scales(b, group):
    # every element and scale of a weight counts on its own
    x = rows_of(b, 513, F32, 3, 2.0)
    w = torch.zeros(520, 513, device="cuda")
    i = torch.arange(513, device="cuda")
    w[i, i] = torch.exp(3.0 * torch.randn(513, generator=generator(4), device="cuda"))
    check_product(x, w, group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("b", [5, 300])
def test_rows_that_are_not_finite_in_a_product(b, group):
    x, w = rows_of(b, 200, F32, 5, 0.3), rows_of(140, 200, F32, 6, 0.3)
    x[3, 7] = float("inf")
    w[130, 199] = float("nan")
    w[5] = 0.0
    check_product(x, w, group)


@pytest.mark.parametrize("group", [16, 32])
def test_strided_products_and_repeats(group):
    x, w = rows_of(150, 400, BF16, 7, 0.3), rows_of(300, 400, BF16, 8, 0.3)
    y, packed = check_product(x[:, 3:260], w[:, 3:260], group)
    check_product(x[::7], w, group)
    check_product(x[:1].expand(140, 400), w[::2], group)
    for _ in range(2):
        assert torch.equal(y, pvs.pvs_mx_matmul(x[:, 3:260], *packed, group))
    # packed rows that start anywhere
    codes, scales, rows = packed
    views = [torch.empty(t.numel() + 3, dtype=t.dtype, device="cuda")[3:].view(t.shape).copy_(t) for t in (codes, scales)]
    assert torch.equal(y, pvs.pvs_mx_matmul(x[:, 3:260], *views, rows, group))


@pytest.mark.parametrize("group", [16, 32])
def test_nothing_to_multiply(group):
    w = rows_of(10, 128, BF16)
    packed = pvs.pvs_mx_pack(w, group)
    assert pvs.pvs_mx_matmul(w[:0], *packed, group).shape == (0, 10)
    none = pvs.pvs_mx_pack(w[:0], group)
    assert pvs.pvs_mx_matmul(w, *none, group).shape == (10, 0)


@pytest.mark.parametrize("b", [4, 300])
def test_in_a_graph_and_on_a_stream(b):
    x, w = rows_of(b, 768, BF16, 9, 0.3), rows_of(1000, 768, BF16, 10, 0.3)
    packed = pvs.pvs_mx_pack(w, 16)
    want = pvs.pvs_mx_matmul(x, *packed, 16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = pvs.pvs_mx_matmul(x, *packed, 16)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = pvs.pvs_mx_matmul(x, *packed, 16)
    x.copy_(rows_of(b, 768, BF16, 11, 0.3))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, pvs.pvs_mx_matmul(x, *packed, 16))


@pytest.mark.parametrize("b", [4, 300])
def test_a_wait_that_runs_out(b):
    x, w = rows_of(b, 768, BF16, 9, 0.3), rows_of(100_000, 768, BF16, 10, 0.3)
    packed = pvs.pvs_mx_pack(w, 32)
    want = pvs.pvs_mx_matmul(x, *packed, 32)
    torch.cuda.synchronize()
    pvs.pvs_head_set_wait_limit(0)
    try:
        pvs.pvs_mx_matmul(x, *packed, 32)
        torch.cuda.synchronize()
        with pytest.raises(pvs.PvsError):
            pvs.pvs_mx_matmul(x, *packed, 32)
    finally:
        pvs.pvs_head_set_wait_limit(2_000_000_000)
    torch.cuda.synchronize()
    pvs.pvs_head_status()
    assert torch.equal(want, pvs.pvs_mx_matmul(x, *packed, 32))


def test_rows_behind_the_outputs_stay():
    x, w = rows_of(5, 128, BF16), rows_of(100, 128, BF16, 1)
    codes, scales, _ = pvs.pvs_mx_pack(w, 32)
    y = torch.full((7, 110), 3.0, dtype=BF16, device="cuda")
    import ctypes
    n = ctypes.c_size_t()
    assert pvs._lib.pvs_mx_workspace(5, 100, 128, 32, ctypes.byref(n)) == pvs.PVS_OK
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    assert pvs._lib.pvs_mx_matmul(x.data_ptr(), 128, 5, codes.data_ptr(), scales.data_ptr(), None, 100, 128, 32,
                                  pvs.PVS_BF16, y.data_ptr(), 110, ws.data_ptr(), n.value,
                                  torch.cuda.current_stream().cuda_stream) == pvs.PVS_OK
    torch.cuda.synchronize()
    assert torch.equal(y[:5, :100], pvs.pvs_mx_matmul(x, codes, scales, None, 32))
    assert (y[5:] == 3.0).all() and (y[:, 100:] == 3.0).all()


def test_refusals():
    x = rows_of(4, 128, BF16)
    codes, scales, rows = pvs.pvs_mx_pack(x, 16)
    for bad, err in (((x, 8), ValueError), ((x.double(), 16), TypeError), ((x[0], 16), ValueError),
                     ((x.cpu(), 16), TypeError)):
        with pytest.raises(err):
            pvs.pvs_mx_pack(*bad)
    for bad, err in (((codes, scales, None, 16), ValueError), ((codes, scales, rows, 32), ValueError),
                     ((codes[:, :32], scales, rows, 16), ValueError), ((codes, scales[:, :1], rows, 16), ValueError),
                     ((codes, scales, rows[:3], 16), ValueError), ((codes.int(), scales, rows, 16), TypeError),
                     ((codes, scales.int(), rows, 16), TypeError), ((codes, scales, rows.double(), 16), TypeError)):
        with pytest.raises(err):
            pvs.pvs_mx_matmul(x, *bad)
        with pytest.raises(err):
            pvs.pvs_mx_unpack(*bad, 128, BF16)
    with pytest.raises(ValueError):
        pvs.pvs_mx_matmul(rows_of(4, 129, BF16), codes, scales, rows, 16)
    with pytest.raises(ValueError):
        pvs.pvs_mx_unpack(codes, scales, rows, 16, 129, BF16)
    with pytest.raises(TypeError):
        pvs.pvs_mx_unpack(codes, scales, rows, 16, 128, torch.float64)
