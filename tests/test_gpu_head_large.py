"""Tables, items and packed rows of more than 2^31 elements: what lies behind that offset."""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
V, D = 2_150_000, 1024
assert V * D > 1 << 31


@pytest.fixture(scope="module")
def table():
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(V, D, dtype=BF16, device="cuda")
    for i in range(0, V, 1 << 18):
        w[i:i + (1 << 18)] = torch.randn(min(1 << 18, V - i), D, generator=g, device="cuda")
    yield w
    del w
    torch.cuda.empty_cache()


def test_lookup_and_gradient(table):
    ids = torch.tensor([0, V - 1, V - 2, 2_097_152, V - 1, 5], device="cuda")
    assert torch.equal(pvs.pvs_embed_forward(table, ids, 2.0), (table[ids].float() * 2.0).to(BF16))
    dy = torch.randn(6, D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(BF16)
    dw = pvs.pvs_embed_backward(dy, ids, V)
    assert torch.equal(dw[V - 2], dy[2]) and torch.equal(dw[2_097_152], dy[3]) and torch.equal(dw[5], dy[5])
    assert torch.equal(dw[V - 1], (dy[1].float() + dy[4].float()).to(BF16))
    dw[ids] = 0
    assert not dw.any()


def test_gradient_of_many_rows(table):
    # more than 2^31 elements on the other side: dy
    ids = torch.arange(V, device="cuda") % 3
    ids[V - 1] = 3
    dw = pvs.pvs_embed_backward(table, ids, 4)
    assert torch.equal(dw[3], table[V - 1])
    part = table[0:V - 1:3]
    want = torch.zeros(D, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for i in range(0, part.shape[0], 1 << 16):
        want += part[i:i + (1 << 16)].double().sum(dim=0)
        size += part[i:i + (1 << 16)].double().abs().sum(dim=0)
    # sums of 32, of an eighth of the pieces, and of eight: about 2,900 roundings of partial sums
    tol = 2.0 ** -9 * want.abs() * 2 + 2_900 * 2.0 ** -24 * size
    assert ((dw[0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("T", [3, 200])
def test_distillation_over_the_last_items(table, T):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = (torch.randn(T, D, generator=g, device="cuda") / D ** 0.5).to(BF16)
    ids = torch.randint(V - 1000, V, (T, 8), generator=g, device="cuda")
    z = torch.randn(T, 8, generator=g, device="cuda")
    loss, stats, hits = pvs.pvs_distill_forward(x, table, ids, z)
    rows = [0, T - 1]
    l = torch.cat([x[rows].double() @ table[i:i + (1 << 18)].double().T for i in range(0, V, 1 << 18)], dim=1)
    logq = l - torch.logsumexp(l, dim=1, keepdim=True)
    logp = torch.log_softmax(z[rows].double(), dim=1)
    want = (logp.exp() * (logp - logq.gather(1, ids[rows]))).sum(dim=1)
    assert ((loss[rows].double() - want).abs() <= 1e-4).all()
    grad = torch.ones(T, device="cuda")
    dx, dw = pvs.pvs_distill_backward(x, table, ids, stats, hits, grad)
    j = ids[0, 0]
    q = torch.exp(x.double() @ table[j].double() - (stats[:, 0].double() * 0.6931471805599453 + stats[:, 1].double().log()))
    p = torch.where(ids == j, torch.softmax(z.double(), dim=1), 0.0).sum(dim=1)
    want = ((q - p)[:, None] * x.double()).sum(dim=0)
    size = ((q + p)[:, None] * x.double().abs()).sum(dim=0)
    # the entry's rounding in two parts, the logits' and the shares' 2^-11, the output's half step
    assert ((dw[j].double() - want).abs() <= 2.0 ** -11 * size + 2.0 ** -8 * want.abs()).all()


@pytest.mark.parametrize("group", [16, 32])
def test_microscaled_rows(table, group):
    codes, scales, rows = pvs.pvs_mx_pack(table, group)
    assert codes.numel() > 1 << 30
    few = pvs.pvs_mx_pack(table[V - 300:], group)
    assert torch.equal(codes[V - 300:], few[0])
    kept = pvs.pvs_mx_unpack(few[0], few[1], few[2], group, D, F32)
    got = pvs.pvs_mx_unpack(codes, scales, rows, group, D, F32)
    assert torch.equal(got[V - 300:], kept)
    del got
    x = table[:5].clone()
    y = pvs.pvs_mx_matmul(x, codes, scales, rows, group)
    assert torch.equal(y[:, V - 300:], pvs.pvs_mx_matmul(x, *few, group))


@pytest.mark.parametrize("T", [3, 200])
def test_distillation_gradients_over_all_items(table, T):
    # both gradients, of items on both sides of the offset, against binary64
    g = torch.Generator(device="cuda").manual_seed(4)
    x = (torch.randn(T, D, generator=g, device="cuda") / D ** 0.5).to(BF16)
    ids = torch.cat([torch.randint(0, 1000, (T, 4), generator=g, device="cuda"),
                     torch.randint(V - 1000, V, (T, 4), generator=g, device="cuda")], dim=1)
    z = torch.randn(T, 8, generator=g, device="cuda")
    grad = torch.rand(T, generator=g, device="cuda") + 0.5
    _, stats, hits = pvs.pvs_distill_forward(x, table, ids, z)
    dx, dw = pvs.pvs_distill_backward(x, table, ids, stats, hits, grad)
    pieces = [(i, min(i + (1 << 18), V)) for i in range(0, V, 1 << 18)]
    X, p, gr = x.double(), torch.softmax(z.double(), dim=1), grad.double()[:, None]
    lse = torch.logsumexp(torch.stack([torch.logsumexp(X @ table[a:b].double().T, dim=1) for a, b in pieces]), dim=0)
    # an entry of G: a logit's steps of 16 and its rounding in a share of q, 2^-20 of p and its
    # exponent's rounding, and 2^-15 for the two parts; a sum: its steps of 16, cut to 24 bits
    e = (D / 16 + 4) * 2.0 ** -23 * 8.0 * float(X.norm(dim=1).max()) * D ** 0.5 + 2.0 ** -19
    t = 2.0 ** -20 + 2.0 ** -22 * 8.0 + 2.0 ** -15
    want, size, off = (torch.zeros(T, D, dtype=torch.float64, device="cuda") for _ in range(3))
    rows = torch.cat([torch.arange(40, device="cuda"), torch.arange(2_097_130, 2_097_170, device="cuda"),
                      torch.arange(V - 40, V, device="cuda"), ids[0], ids[T - 1]])
    for a, b in pieces:
        W = table[a:b].double()
        q = torch.exp(X @ W.T - lse[:, None]) * gr
        here = (ids >= a) & (ids < b)
        P = torch.zeros_like(q).scatter_add_(1, (ids - a).clamp(0, b - a - 1), torch.where(here, p, 0.0) * gr)
        want += (q - P) @ W
        size += (q + P) @ W.abs()
        off += ((2 * e + 2.0 ** -15) * q + t * P) @ W.abs()
        j = rows[(rows >= a) & (rows < b)]
        if len(j):
            G = (q - P)[:, j - a].T
            to = G @ X
            slack = (((2 * e + 2.0 ** -15) * q + t * P)[:, j - a].T + (T / 16 + 8) * 2.0 ** -23 * G.abs()) @ X.abs()
            assert ((dw[j].double() - to).abs() <= slack + 2.0 ** -8 * to.abs() + 2.0 ** -126).all()
    tol = off + (V / 16 + 8) * 2.0 ** -23 * size + 2.0 ** -8 * want.abs()
    assert ((dx.double() - want).abs() <= tol).all()
    # (the bound is far below the gradients: items that were not read would show)
    assert float(tol.norm()) < 0.1 * float(want.norm())
