"""Table lookups and the table's gradient against the definition in binary64.

Tolerances, taken before any run: a looked-up row is the float32 product rounded to its
type, to the bit.  A sum of c float32 terms rounds c - 1 times, its scaling once more and the
output once: (c + 1) 2^-24 of the sum of the terms' sizes, and half a step of the output.
"""
import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25, F32: 2.0 ** -149}
IGNORE = -100


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def some_ids(n, V, how, seed=0):
    g = generator(seed)
    if how == "same":
        return torch.full((n,), V - 1, device="cuda")
    if how == "none":
        return torch.full((n,), IGNORE, device="cuda")
    if how == "down":
        return torch.arange(n, 0, -1, device="cuda") % V
    if how == "few":
        return torch.randint(0, min(V, 3), (n,), generator=g, device="cuda")
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    if how == "mixed":
        ids[torch.rand(n, generator=g, device="cuda") < 0.2] = IGNORE
        ids[torch.rand(n, generator=g, device="cuda") < 0.1] = V
        ids[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
        ids[torch.rand(n, generator=g, device="cuda") < 0.3] = V // 2
    return ids


def check_lookup(w, ids, scale, **kw):
    y = pvs.pvs_embed_forward(w, ids, scale=scale, **kw)
    ignore = kw.get("ignore_index", IGNORE)
    out = (ids < 0) | (ids >= w.shape[0])
    want = w[torch.where(out, 0, ids)].float() * torch.tensor(scale, dtype=F32, device="cuda")
    want[out] = float("nan")
    want[ids == ignore] = 0.0
    want = want.to(w.dtype)
    assert y.dtype == w.dtype and y.shape == want.shape
    assert torch.equal(torch.nan_to_num(y.float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0))


def check_gradient(dy, ids, V, scale, **kw):
    dw = pvs.pvs_embed_backward(dy, ids, V, scale=scale, **kw)
    kept = (ids >= 0) & (ids < V) & (ids != kw.get("ignore_index", IGNORE))
    at, rows = ids[kept], dy[kept].double()
    want = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, rows) * scale
    size = torch.zeros_like(want).index_add_(0, at, rows.abs()) * abs(scale)
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    tol = (count[:, None] + 1) * 2.0 ** -24 * size + torch.finfo(dy.dtype).eps / 2 * want.abs() * (1 + 2.0 ** -20)
    tol = tol + TINY[dy.dtype]
    assert dw.dtype == dy.dtype and dw.shape == want.shape
    over = (dw.double() - want).abs() > tol
    assert not over.any(), (int(over.sum()), float((dw.double() - want).abs()[over].max()))
    again = pvs.pvs_embed_backward(dy, ids, V, scale=scale, **kw)
    assert torch.equal(dw, again)
    return dw


SHAPES = [(1, 1, 1), (1, 50_000, 768), (31, 2, 7), (32, 77, 8), (33, 77, 264), (64, 5, 256), (65, 1023, 100),
          (1000, 1024, 385), (4096, 1025, 72), (4097, 1025, 72), (8192, 300, 72), (8193, 70_000, 264), (6000, 1 << 20, 24), (10_000, 600, 33),
          (70_000, 50_000, 16), (300, 100, 2056), (200, 9, 32_767)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,V,d", SHAPES)
def test_lookup_and_gradient(n, V, d, dtype):
    g = generator(1)
    w = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    dy = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    for how in ("any", "mixed"):
        ids = some_ids(n, V, how)
        check_lookup(w, ids, 27.7)
        check_gradient(dy, ids, V, 27.7)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 31, 32, 33, 34, 64, 65, 95, 2500, 9000, 40_000])
@pytest.mark.parametrize("how", ["same", "none", "down", "few"])
def test_runs_of_one_id(n, how):
    dy = torch.randn(n, 40, generator=generator(2), device="cuda")
    for dtype, V in ((F32, 5), (BF16, 3000)):
        check_gradient(dy.to(dtype), some_ids(n, V, how), V, -0.5)


@pytest.mark.parametrize("n", [3000, 41_000])
@pytest.mark.parametrize("seed", range(3))
def test_runs_of_every_length(n, seed):
    # runs of 1 to 100 entries, so that they start, cross and end everywhere in the pieces
    g = generator(100 + seed)
    lengths = torch.randint(1, 101, (n // 40,), generator=g, device="cuda")
    ids = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda") * 2, lengths)[:n]
    dy = torch.randn(ids.numel(), 24, generator=g, device="cuda")
    V = 2 * lengths.numel()
    check_gradient(dy, ids, V, 1.0)
    check_gradient(dy.to(BF16), ids[torch.randperm(ids.numel(), generator=g, device="cuda")], V, 1.0)


def test_long_run_amid_others():
    # a run over hundreds of pieces, with neighbours on both sides
    ids = torch.cat([torch.arange(50, device="cuda"), torch.full((20_000,), 50, device="cuda"),
                     torch.arange(51, 100, device="cuda")])
    dy = torch.randn(ids.numel(), 136, generator=generator(3), device="cuda")
    check_gradient(dy, ids[torch.randperm(ids.numel(), generator=generator(4), device="cuda")], 100, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_and_unaligned(dtype):
    g = generator(5)
    w = torch.randn(300, 200, generator=g, device="cuda").to(dtype)
    dy = torch.randn(500, 200, generator=g, device="cuda").to(dtype)
    ids = some_ids(500, 300, "mixed")
    for lo, hi in ((0, 96), (1, 97), (3, 200), (8, 72)):
        check_lookup(w[:, lo:hi], ids, 2.0)
        check_gradient(dy[:, lo:hi], ids, 300, 2.0)
    check_lookup(w.T.contiguous().T, ids, 2.0)
    check_gradient(dy[::2], ids[::2], 300, 2.0)
    check_lookup(w[::3], ids[::5] % 100, 1.0)
    check_gradient(dy[:1].expand(500, 200), ids, 300, 2.0)


def test_other_ignored_ids_and_no_rows():
    w = torch.randn(10, 16, generator=generator(6), device="cuda")
    ids = torch.tensor([0, 3, 3, 9, 0], device="cuda")
    check_lookup(w, ids, 1.0, ignore_index=3)
    check_gradient(w[:5], ids, 10, 1.0, ignore_index=3)
    none = ids[:0]
    assert pvs.pvs_embed_forward(w, none).shape == (0, 16)
    assert not pvs.pvs_embed_backward(w[:0], none, 10).any()


def test_rows_without_a_place_may_hold_anything():
    dy = torch.full((40, 24), float("nan"), device="cuda")
    ids = torch.full((40,), IGNORE, device="cuda")
    ids[7], ids[8] = 2, 99
    dy[7] = 1.5
    dw = pvs.pvs_embed_backward(dy, ids, 6)
    want = torch.zeros(6, 24, device="cuda")
    want[2] = 1.5
    assert torch.equal(dw, want)
    # infinities reach their own rows alone
    dy[7, 3] = float("inf")
    assert torch.equal(torch.isinf(pvs.pvs_embed_backward(dy, ids, 6)).nonzero(), torch.tensor([[2, 3]], device="cuda"))


def test_gradient_by_differences():
    # the gradient of sum(c y) by the table's entries, which the lookup is linear in
    g = generator(7)
    w = torch.randn(7, 5, generator=g, device="cuda")
    c = torch.randn(20, 5, generator=g, device="cuda")
    ids = some_ids(20, 7, "any")
    dw = pvs.pvs_embed_backward(c, ids, 7, scale=3.0)
    for v in range(7):
        for k in range(5):
            up = w.clone()
            up[v, k] += 1.0
            up[v, k] = up[v, k]
            step = (up[v, k] - w[v, k]).double()
            d = (pvs.pvs_embed_forward(up, ids, 3.0).double() - pvs.pvs_embed_forward(w, ids, 3.0).double()) * c.double()
            # each difference of two rounded products is off by 2^-24 of both of them
            tol = 2.0 ** -23 * 3.0 * (w[v, k].abs() + 1.0) * 2 * c[:, k].abs().sum() + 2.0 ** -20 * dw[v, k].abs()
            assert abs(float(d.sum() / step - dw[v, k])) <= float(tol) + 1e-12


def test_on_a_stream_and_in_a_graph():
    g = generator(8)
    w = torch.randn(900, 64, generator=g, device="cuda").to(BF16)
    dy = torch.randn(5000, 64, generator=g, device="cuda").to(BF16)
    ids = some_ids(5000, 900, "mixed")
    want_y, want = pvs.pvs_embed_forward(w, ids, 2.0), pvs.pvs_embed_backward(dy, ids, 900, 2.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y, dw = pvs.pvs_embed_forward(w, ids, 2.0), pvs.pvs_embed_backward(dy, ids, 900, 2.0)
    s.synchronize()
    assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(want_y)) and torch.equal(dw, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dw = pvs.pvs_embed_forward(w, ids, 2.0), pvs.pvs_embed_backward(dy, ids, 900, 2.0)
    for seed in (9, 10):
        ids.copy_(some_ids(5000, 900, "mixed", seed))
        dy.copy_(torch.randn(5000, 64, generator=generator(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(pvs.pvs_embed_forward(w, ids, 2.0)))
        assert torch.equal(dw, pvs.pvs_embed_backward(dy, ids, 900, 2.0))


def test_rows_behind_the_outputs_stay():
    # through the C boundary: a leading dimension larger than the row
    w = torch.randn(40, 24, generator=generator(11), device="cuda")
    ids = some_ids(100, 40, "any")
    y = torch.full((102, 30), 7.0, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    assert pvs._lib.pvs_embed_forward(w.data_ptr(), 24, 40, 24, pvs.PVS_F32, ids.data_ptr(), 100, 1.0, IGNORE,
                                      y.data_ptr(), 30, st) == pvs.PVS_OK
    torch.cuda.synchronize()
    assert torch.equal(y[:100, :24], w[ids]) and (y[100:] == 7.0).all() and (y[:, 24:] == 7.0).all()


def test_refusals():
    w = torch.zeros(4, 8, device="cuda")
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        pvs.pvs_embed_forward(w, ids.int())
    with pytest.raises(TypeError):
        pvs.pvs_embed_forward(w.double(), ids)
    with pytest.raises(TypeError):
        pvs.pvs_embed_forward(w, ids.cpu())
    with pytest.raises(ValueError):
        pvs.pvs_embed_forward(w, ids[None])
    with pytest.raises(ValueError):
        pvs.pvs_embed_forward(w[:0], ids)
    with pytest.raises(ValueError):
        pvs.pvs_embed_forward(w, ids, scale=float("inf"))
    with pytest.raises(ValueError):
        pvs.pvs_embed_backward(w, ids, 10)
    with pytest.raises(ValueError):
        pvs.pvs_embed_backward(w[:3], ids, 0)
