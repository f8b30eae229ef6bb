"""Distillation from a teacher's best logits and its gradients against the definition in
binary64.

Tolerances are bounds on the rounding of the kernels, taken before any run.  A logit of d
products summed in float32 steps of 16 is off by at most e = (d / 16 + 4) 2^-23 a sum|x w| +
2^-22 |l| (sums may be cut, not rounded).  A teacher's share is off by t = 2^-20 + 2^-22 max|c z|
of itself (the scaled logit's rounding in the exponent, the exponential, the sum of K of them and
the division).  A loss: 2 e + 2^-19 for the logarithms of the student's shares, and (t + 2^-21) sum_k
p_k (|ln p_k| + |ln q_k| + 1).  An entry g (q - p) of G: its type's rounding, 2 e + 2^-19 of q
and t of p, and 2^-23 of both; a gradient by that through sum|G w|, its own steps, and its type's
rounding.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 2.0 ** -126, F16: 2.0 ** -24, F32: 2.0 ** -126}
INF = math.inf
IGNORE = -100


def make(T, V, d, K, dtype, seed=0, masked=0.0, empty=0.0, spread=4.0, teacher=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(T, d, generator=g, device="cuda") / d ** 0.5).to(dtype)
    w = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    ids = torch.randint(0, V, (T, K), generator=g, device="cuda")
    z = (2.0 * torch.randn(T, K, generator=g, device="cuda")).to(teacher)
    bias = None
    if masked:
        bias = torch.randn(V, generator=g, device="cuda")
        bias[torch.rand(V, generator=g, device="cuda") < masked] = -INF
    if empty:
        ids[torch.rand(T, K, generator=g, device="cuda") < empty] = IGNORE
        z[torch.rand(T, K, generator=g, device="cuda") < empty / 2] = -INF
        ids[torch.rand(T, generator=g, device="cuda") < empty] = IGNORE
    grad = torch.randn(T, generator=g, device="cuda") / T
    return dict(x=x, w=w, ids=ids, z=z, bias=bias, grad=grad, scale=spread, c=0.75)


def reference(x, w, ids, z, bias, grad, scale, c):
    """loss, dx, dw of the definition in binary64, and their tolerances."""
    X, W = x.double(), w.double()
    d, V = X.shape[1], W.shape[0]
    out = torch.zeros(V, dtype=torch.bool, device=x.device)
    if bias is not None:
        out = bias == -INF
    at = ids.clamp(0, V - 1)
    listed = (ids != IGNORE) & ~out[at] & (z != -INF)
    dead = ~listed.any(dim=1)
    W0 = torch.where(out[:, None], 0.0, W)
    X0 = torch.where(dead[:, None], 0.0, X)
    l = scale * (X0 @ W0.T)
    if bias is not None:
        l = l + bias.double()
    lse = torch.logsumexp(l, dim=1)
    lse = torch.where(torch.isfinite(lse), lse, 0.0)
    cz = (c * z.double()).masked_fill(~listed, -INF)
    log_p = cz - torch.where(dead, 0.0, torch.logsumexp(cz, dim=1))[:, None]
    p = torch.exp(log_p)
    log_q = l.gather(1, at) - lse[:, None]
    terms = torch.where(listed, p * (log_p - log_q), 0.0)
    loss = terms.sum(dim=1)
    q = torch.where(dead[:, None], 0.0, torch.exp(l - lse[:, None]))
    P = torch.zeros_like(q).scatter_add_(1, at, p)
    g = grad.double()[:, None]
    G = (q - P) * g
    size = scale * (X0.abs() @ W0.abs().T)
    lf = torch.where(torch.isfinite(l), l.abs(), 0.0)
    e = ((d / 16 + 4) * 2.0 ** -23 * size + 2.0 ** -22 * lf).amax(dim=1)
    t = 2.0 ** -20 + 2.0 ** -22 * torch.where(listed, cz.abs(), 0.0).amax(dim=1)
    spread = torch.where(listed, p * (log_p.abs() + log_q.abs() + 1.0), 0.0).sum(dim=1)
    tol_loss = 2 * e + 2.0 ** -19 + (t + 2.0 ** -21) * spread
    unit = UNIT[x.dtype]
    A = (unit * (q - P).abs() + (2 * e + 2.0 ** -19)[:, None] * q + t[:, None] * P + 2.0 ** -23 * (q + P)) * g.abs()
    if x.dtype == F16:   # entries below the scaled f16's last bit
        A = A + grad.abs().max().double() * 2.0 ** -37
    dx, dw = scale * (G @ W0), scale * (G.T @ X0)
    aG = G.abs()
    tdx = scale * (A @ W0.abs()) + (V / 16 + 8) * 2.0 ** -23 * scale * (aG @ W0.abs())
    tdw = scale * (A.T @ X0.abs()) + (X.shape[0] / 16 + 8) * 2.0 ** -23 * scale * (aG.T @ X0.abs())
    tdx = tdx + unit * dx.abs() + TINY[x.dtype]
    tdw = tdw + unit * dw.abs() + TINY[x.dtype]
    return (loss, dx, dw), (tol_loss, tdx, tdw)


def close(got, want, tol):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got - want).abs()[fine]
    over = off > tol.expand_as(want)[fine]
    assert not over.any(), (float(off[over].max()), int(over.sum()), off.numel())


def step(x, w, ids, z, bias, grad, scale, c, **kw):
    loss, stats, hits = pvs.pvs_distill_forward(x, w, ids, z, bias=bias, scale=scale, teacher_scale=c)
    dx, dw = pvs.pvs_distill_backward(x, w, ids, stats, hits, grad, bias=bias, scale=scale, **kw)
    return loss, dx, dw


def check(case):
    got = step(**case)
    want, tol = reference(**case)
    for a, b, t in zip(got, want, tol):
        assert a.dtype in (case["x"].dtype, F32)
        close(a, b, t)
    torch.cuda.synchronize()
    assert pvs.pvs_head_status() == pvs.PVS_OK
    return got


SHAPES = [(1, 1, 1, 1), (1, 2, 3, 5), (2, 17, 8, 2), (1, 10_000, 128, 33), (127, 255, 64, 16), (128, 256, 256, 31),
          (129, 257, 65, 32), (300, 1000, 385, 100), (33, 4097, 768, 1024), (1000, 100, 1024, 7), (5, 70_001, 24, 64),
          (4096, 300, 40, 3), (257, 999, 513, 999), (16, 513, 2000, 129), (700, 2000, 128, 513)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,d,K", SHAPES)
def test_step_matches_definition(T, V, d, K, dtype):
    check(make(T, V, d, K, dtype))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V,d,K", [(1, 300, 16, 4), (200, 777, 136, 20), (130, 3000, 385, 200)])
@pytest.mark.parametrize("masked,empty", [(0.5, 0.0), (0.02, 0.3), (0.97, 0.9)])
def test_masks_and_short_lists(T, V, d, K, masked, empty, dtype):
    check(make(T, V, d, K, dtype, masked=masked, empty=empty))


@pytest.mark.parametrize("teacher", [BF16, F16])
def test_teacher_types(teacher):
    check(make(70, 500, 64, 12, BF16, teacher=teacher, empty=0.1))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_several_pieces_of_the_vocabulary(dtype):
    # the gradient of every logit would be 0.5 to 1.6 GB here: several pieces
    check(make(8192, 33_001, 24, 40, dtype, masked=0.1, empty=0.1))


@pytest.mark.parametrize("T", [3, 40])
def test_several_pieces_of_copied_items(T):
    # float32 items are copied 1 GB at a time: three pieces of the forward pass (few rows: one)
    check(make(T, 400_000, 1000, 24, F32, masked=0.05, empty=0.1))


def test_several_blocks_of_rows():
    # 8 bytes of statistics for each row and 256 items: two blocks of the forward pass
    case = make(2100, 16_900_000, 8, 5, BF16, empty=0.1)
    loss, stats, hits = pvs.pvs_distill_forward(case["x"], case["w"], case["ids"], case["z"], scale=case["scale"],
                                                teacher_scale=case["c"])
    for r in (0, 1023, 2047, 2048, 2099):
        one = {k: (v[r:r + 1] if k in ("x", "ids", "z", "grad") else v) for k, v in case.items()}
        (want, _, _), (tol, _, _) = reference(**one)
        close(loss[r:r + 1], want, tol)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_strided_and_unaligned_operands(dtype):
    case = make(70, 501, 96, 9, dtype)
    for d, off in ((96, 0), (90, 3), (33, 1)):
        xs = torch.full((70, 140), float("nan"), dtype=dtype, device="cuda")
        ws = torch.full((501, 123), float("nan"), dtype=dtype, device="cuda")
        xs[:, off:off + d] = case["x"][:, :d]
        ws[:, off:off + d] = case["w"][:, :d]
        check(dict(case, x=xs[:, off:off + d], w=ws[:, off:off + d]))
    check(dict(case, x=case["x"].T.contiguous().T, w=case["w"].T.contiguous().T))
    check(dict(case, ids=case["ids"].T.contiguous().T, z=case["z"].T.contiguous().T))
    check(dict(case, x=case["x"][:1].expand(70, 96), ids=case["ids"][:1].expand(70, 9)))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T", [3, 40])
def test_the_same_item_twice(T, dtype):
    case = make(T, 300, 64, 24, dtype)
    case["ids"] %= 5
    case["ids"][0] = 7
    case["ids"][1, ::2] = 299
    check(case)


@pytest.mark.parametrize("T", [3, 40])
def test_one_slot_is_the_cross_entropy(T):
    case = make(T, 300, 64, 1, F32)
    loss, dx, dw = check(case)
    want, stats = pvs.pvs_xent_forward(case["x"], case["w"], case["ids"][:, 0], scale=case["scale"])
    _, tol = reference(**case)
    close(loss, want.double(), 2 * tol[0])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T", [5, 50])
def test_rows_without_a_list_and_bad_ids(T, dtype):
    case = make(T, 200, 40, 6, dtype)
    case["ids"][1] = IGNORE
    case["x"][1] = float("nan")
    loss, dx, dw = check(case)
    assert loss[1] == 0 and not dx[1].any()
    # an id outside the items: its row is NaN, and what that reaches
    case["x"][1] = 0.0
    case["ids"][3, 2] = 200
    loss, dx, dw = step(**case)
    assert torch.isnan(loss).nonzero().tolist() == [[3]]
    assert torch.isnan(dx).any(dim=1).nonzero().tolist() == [[3]] and torch.isnan(dw).all()
    case["ids"][3, 2] = -7
    assert torch.isnan(step(**case)[0][3])


@pytest.mark.parametrize("T", [5, 50])
def test_every_item_masked(T):
    case = make(T, 100, 32, 4, BF16)
    case["bias"] = torch.full((100,), -INF, device="cuda")
    case["w"][3] = float("nan")
    loss, dx, dw = step(**case)
    assert not loss.any() and not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [5, 50])
def test_masked_items_may_hold_anything(T, dtype):
    case = make(T, 400, 64, 8, dtype, masked=0.2)
    out = (case["bias"] == -INF).nonzero()[:, 0]
    case["ids"][:, 0] = out[0]
    check(case)
    case["w"][out[::3]] = float("nan")
    case["w"][out[1::3]] = INF
    got = step(**case)
    case["w"][out] = 0.0
    for a, b, t in zip(got, *reference(**case)):
        close(a, b, t)


@pytest.mark.parametrize("T", [5, 50])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_biases_of_the_lowest_value(T, dtype):
    # a mask by the type's lowest value: those items have no share, and lists without them keep their loss
    case = make(T, 300, 64, 6, dtype)
    case["bias"] = torch.zeros(300, device="cuda")
    case["bias"][200:] = torch.finfo(F32).min
    case["ids"] %= 200
    got = step(**case)
    hidden = dict(case, bias=case["bias"].clone())
    hidden["bias"][200:] = -INF
    for a, b, t in zip(got, *reference(**hidden)):
        close(a, b, t)


@pytest.mark.parametrize("limit_first", [True, False])
def test_a_wait_that_runs_out(limit_first):
    case = make(300, 20_000, 512, 8, BF16)
    want = step(**case)
    loss, stats, hits = pvs.pvs_distill_forward(case["x"], case["w"], case["ids"], case["z"], scale=case["scale"],
                                                teacher_scale=case["c"])
    torch.cuda.synchronize()
    pvs.pvs_head_set_wait_limit(0)
    try:
        if limit_first:
            pvs.pvs_distill_forward(case["x"], case["w"], case["ids"], case["z"])
        else:
            pvs.pvs_distill_backward(case["x"], case["w"], case["ids"], stats, hits, case["grad"])
        torch.cuda.synchronize()
        with pytest.raises(pvs.PvsError):
            pvs.pvs_head_status()
    finally:
        pvs.pvs_head_set_wait_limit(2_000_000_000)
    assert all(torch.equal(a, b) for a, b in zip(want, step(**case)))


def test_nan_and_infinite_teacher():
    case = make(40, 300, 32, 5, BF16)
    case["z"][2, 1] = float("nan")
    case["z"][3, 1] = INF
    loss, dx, dw = step(**case)
    assert torch.isnan(loss).nonzero().flatten().tolist() == [2, 3]
    assert torch.isnan(dx).any(dim=1).nonzero().flatten().tolist() == [2, 3]


@pytest.mark.parametrize("T", [4, 30])
def test_gradient_by_differences(T):
    case = make(T, 60, 16, 5, F32, masked=0.1, empty=0.1)
    case["grad"] = case["grad"].abs() + 0.1
    _, dx, dw = step(**case)
    g = torch.Generator(device="cuda").manual_seed(5)
    for name, grad in (("x", dx), ("w", dw)):
        v = torch.randn(case[name].shape, generator=g, device="cuda")
        h = 2.0 ** -10
        # the definition's own losses on both sides (its loss is held to the kernel's above)
        up = reference(**dict(case, **{name: case[name].double() + h * v.double(), **wide(case, name)}))[0][0]
        dn = reference(**dict(case, **{name: case[name].double() - h * v.double(), **wide(case, name)}))[0][0]
        slope = float(((up - dn) * case["grad"].double()).sum() / (2 * h))
        size = float((grad.double() * v.double()).abs().sum())
        # central differences are off by h^2 / 6 of a third derivative, below (a |x| |v|)^3
        assert abs(slope - float((grad.double() * v.double()).sum())) <= 1e-3 * size


def wide(case, name):
    UNIT[torch.float64] = TINY[torch.float64] = 2.0 ** -53
    return {"w" if name == "x" else "x": case["w" if name == "x" else "x"].double()}


def test_parts_alone_and_repeats():
    case = make(300, 5000, 128, 20, BF16, masked=0.05, empty=0.1)
    loss, dx, dw = step(**case)
    for _ in range(2):
        again = step(**case)
        assert all(torch.equal(a, b) for a, b in zip((loss, dx, dw), again))
    only = step(**case, need_w=False)
    assert only[2] is None and torch.equal(only[0], loss)
    close(only[1], *[r[1] for r in reference(**case)])
    only = step(**case, need_x=False)
    assert only[1] is None
    close(only[2], *[r[2] for r in reference(**case)])


def test_in_a_graph_and_on_a_stream():
    case = make(200, 3000, 96, 10, BF16, masked=0.05, empty=0.1)
    want = step(**case)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(**case)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(**case)
    other = make(200, 3000, 96, 10, BF16, seed=3, masked=0.05, empty=0.1)
    for k in ("x", "w", "ids", "z", "bias", "grad"):
        case[k].copy_(other[k])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, step(**other)))


def test_refusals():
    c = make(6, 20, 8, 4, BF16)
    fwd = lambda **kw: pvs.pvs_distill_forward(*[kw.get(n, c[n]) for n in ("x", "w", "ids", "z")],   # noqa: E731
                                               **{k: v for k, v in kw.items() if k not in c or k == "bias" or k == "scale"})
    for kw, err in ((dict(x=c["x"].float()), TypeError), (dict(w=c["w"][:, :4]), ValueError),
                    (dict(ids=c["ids"].int()), TypeError), (dict(ids=c["ids"][:5]), ValueError),
                    (dict(z=c["z"][:, :3]), ValueError), (dict(z=c["z"].double()), TypeError),
                    (dict(z=None), TypeError), (dict(ids=c["ids"][:, :0], z=c["z"][:, :0]), ValueError),
                    (dict(ids=c["ids"].repeat(1, 300), z=c["z"].repeat(1, 300)), ValueError),
                    (dict(scale=0.0), ValueError), (dict(teacher_scale=-1.0), ValueError),
                    (dict(teacher_scale=INF), ValueError), (dict(bias=torch.zeros(19, device="cuda")), ValueError),
                    (dict(w=c["w"][:0]), ValueError), (dict(x=c["x"].cpu()), TypeError)):
        with pytest.raises(err):
            fwd(**kw)
    _, stats, hits = fwd()
    with pytest.raises(ValueError):
        pvs.pvs_distill_backward(c["x"], c["w"], c["ids"], stats, hits[:, :3], c["grad"])
    with pytest.raises(ValueError):
        pvs.pvs_distill_backward(c["x"], c["w"], c["ids"], stats[:5], hits, c["grad"])
    loss, stats, hits = pvs.pvs_distill_forward(c["x"][:0], c["w"], c["ids"][:0], c["z"][:0])
    assert loss.shape == (0,) and hits.shape == (0, 4)
    dx, dw = pvs.pvs_distill_backward(c["x"][:0], c["w"], c["ids"][:0], stats, hits, c["grad"][:0])
    assert dx.shape == (0, 8) and not dw.any()
