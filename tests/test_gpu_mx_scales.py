"""Products and rows of microscaled codes whose sizes are far apart, against the definition in binary64.

An output is rounded once, from a sum of exact products of codes and group scales times the row
scales: it has to be right wherever it is a float32, whatever either row scale does to the sum
alone.  The sum is off by (K / 64 + 8) 2^-23 of sum|x w| (steps of 64, cut to 24 bits), two products
with scales by 2^-23 of the output, its own rounding by half a step of its type, or of its
smallest number.  Groups of 32 have their scales in the tensor cores' steps: each may also be cut to
a whole number of the smallest float32s, and is infinite (and NaN with an infinity of the other
sign) where it leaves float32's range.
"""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
SMALLEST = {BF16: 2.0 ** -133, F16: 2.0 ** -24, F32: 2.0 ** -149}
# rows of both, lone CTAs and pairs; few columns, and as many as are split
SIZES = [(5, 300, 771), (5, 300, 4096), (300, 300, 771), (300, 300, 4096), (150, 20_000, 512)]


def rows_of(r, k, dtype, seed, exponents):
    """Rows of about 1, by turns times powers of two."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(r, k, generator=g, device="cuda") * torch.exp(0.3 * torch.randn(r, 1, generator=g, device="cuda"))
    e = torch.tensor(exponents, device="cuda")[torch.arange(r, device="cuda") % len(exponents)]
    return torch.ldexp(x.clamp(-8.0, 8.0).double(), e[:, None]).to(dtype)


def stands_for(packed, group, k):
    """What packed rows stand for, in binary64: from rows unpacked without their row scales."""
    codes, scales, rows = packed
    one = None if rows is None else torch.ones_like(rows)
    v = pvs.pvs_mx_unpack(codes, scales, one, group, k, F32).double()
    return v if rows is None else v * rows.double()[:, None]


def check(x, packed, group):
    k = x.shape[1]
    y = pvs.pvs_mx_matmul(x, *packed, group)
    X, W = stands_for(pvs.pvs_mx_pack(x, group), group, k), stands_for(packed, group, k)
    want, size = X @ W.T, X.abs() @ W.abs().T
    most = torch.finfo(y.dtype).max
    steps = k / 64 + 8
    off = steps * 2.0 ** -23 * size
    tol = off + (torch.finfo(y.dtype).eps / 2 + 2.0 ** -23) * want.abs() + SMALLEST[y.dtype] / 2
    # an output near the type's largest number may be either, and so may one that the sum's own error
    # takes there; and in groups of 32 one whose float32 sum may leave the range on its way
    beyond = want.abs() > 4.0 * most
    assert not (~beyond & (want.abs() > most / 4.0)).any()
    either = off > torch.where(beyond, want.abs() / 4.0, most / 4.0)
    if group == 32:
        tol = tol + steps * 2.0 ** -149
        assert not torch.isfinite(y[beyond & ~either]).any()
        either |= size > most / 4.0
    must = beyond & ~either
    assert torch.equal(y[must].double(), torch.sign(want[must]) * float("inf"))
    over = ((y.double() - want).abs() > tol) | ~torch.isfinite(y)
    over &= ~beyond & ~either
    assert not over.any(), (int(over.sum()), y.numel(), want[over][:5].tolist(), y[over][:5].tolist())
    assert (must | (~beyond & ~either)).any()
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n,k", SIZES)
def test_rows_of_unlike_sizes(b, n, k, dtype, group):
    # large weights and small rows, the reverse, both large (infinite outputs), both small (zeros)
    w = rows_of(n, k, dtype, 1, [-116, 116, -50, 0, 20]) * k ** -0.5
    x = rows_of(b, k, dtype, 2, [100, -100, -50, 0, -25])
    # (no sum of w's rows by x's may come near the largest float32: 116 + 0 and 20 + 100 stay below 2^125)
    check(x, pvs.pvs_mx_pack(w.to(dtype), group), group)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("b,n", [(5, 300), (300, 300)])
def test_large_weights_of_one_sign(b, n, group):
    # sums of 4,096 terms of one sign, times 2^100, are infinite before the rows' 2^-90
    w = torch.full((n, 4096), 2.0 ** 110, device="cuda") * (1.0 + torch.arange(n, device="cuda")[:, None] / n)
    x = torch.full((b, 4096), 2.0 ** -80, device="cuda") * (1.0 + torch.arange(b, device="cuda")[:, None] / b)
    check(x, pvs.pvs_mx_pack(w, group), group)
    check(w, pvs.pvs_mx_pack(x, group), group)


@pytest.mark.parametrize("b,n,k", SIZES)
def test_row_scales_of_the_callers(b, n, k):
    # scales that no packer makes: below the smallest normal number, no powers of two, negative, zero
    w = rows_of(n, k, F32, 3, [-116, 0, 80])
    codes, scales, rows = pvs.pvs_mx_pack(w, 16)
    for factor, exponents in ((2.0 ** -22, [100, 110]), (1.37, [-60, -20]), (-1.1 * 2.0 ** 50, [-100, -55])):
        r = rows * factor
        r[7] = 0.0
        check(rows_of(b, k, F32, 4, exponents), (codes, scales, r), 16)


@pytest.mark.parametrize("b", [3, 300])
def test_f16_outputs_of_large_weights(b):
    # f16 rows times weights packed in float32: outputs are f16 however large the weights' scales are
    w = rows_of(260, 771, F32, 5, [-20, 0, 4])
    codes, scales, rows = pvs.pvs_mx_pack(w, 16)
    x = rows_of(b, 771, F16, 6, [-10, -3, 0])
    check(x, (codes, scales, torch.ldexp(rows, torch.tensor(-2, device="cuda"))), 16)
    # (2^110 and the rows' own 2^-14 to 2^-24: every output is infinite, or nothing)
    check(x, (codes, scales, torch.ldexp(rows, torch.tensor(110, device="cuda"))), 16)


@pytest.mark.parametrize("k", [128, 385])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_unpacked_rows_of_callers_scales(k, dtype):
    # a code's value times its group's scale is exact: one product, rounded to float32, and its rounding
    x = rows_of(200, k, F32, 7, [0])
    x[:, 32:48] = 0.0                        # (a group of zeros, and codes of zero beside large ones)
    x[:, 50] *= 2.0 ** 12
    codes, scales, rows = pvs.pvs_mx_pack(x, 16)
    units = stands_for((codes, scales, torch.ones_like(rows)), 16, k)
    r = torch.ldexp(rows, torch.tensor([-140, -126, -100, 0, 100, 119, 126], device="cuda")[torch.arange(200, device="cuda") % 7])
    r[3] = 3.4e38
    r[11] = -1.3 * 2.0 ** -145
    want = (units * r.double()[:, None]).float().to(dtype)
    got = pvs.pvs_mx_unpack(codes, scales, r, 16, k, dtype)
    # (some of those scales are infinite: codes of zero are NaN there, and nowhere else)
    bad = torch.isinf(r)[:, None] & (units == 0.0)
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], want[~bad])
