"""Lookups, distillation and microscaled products together, as the example runs them."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pvs = pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_head", os.path.join(ROOT, "examples", "distill_head.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_example_runs(example):
    r = example.run(items_n=3000, steps=5, queries=5, batch=64)
    assert all(v == v for v in r.values())


@pytest.mark.parametrize("masked", [False, True])
def test_gradients_of_the_whole_head(example, masked):
    # against automatic differentiation of the plain formulas in binary64
    head = example.Head(40, 24, 16, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    items = torch.randn(500, 16, generator=g, device="cuda")
    items = items / items.norm(dim=1, keepdim=True)
    tokens = torch.randint(0, 40, (50, 6), generator=g, device="cuda")
    tokens[torch.rand(50, 6, generator=g, device="cuda") < 0.2] = example.EMPTY
    ids = torch.randint(0, 500, (50, 8), generator=g, device="cuda")
    scores = torch.rand(50, 8, generator=g, device="cuda")
    ids[torch.rand(50, 8, generator=g, device="cuda") < 0.1] = example.EMPTY
    ids[3] = example.EMPTY
    bias = None
    if masked:
        bias = torch.zeros(500, device="cuda")
        bias[torch.rand(500, generator=g, device="cuda") < 0.1] = -float("inf")
    head.w *= 0.2
    loss, dtable, dw = head.gradients(tokens, items, ids, scores, bias=bias)

    table, w = head.table.double().requires_grad_(), head.w.double().requires_grad_()
    there = tokens != example.EMPTY
    rows = table[tokens.clamp(min=0)] * there[..., None]
    x = rows.sum(dim=1) * 6 ** -0.5
    l = example.SCALE * (x @ w.T) @ items.double().T
    if masked:
        l = l + bias.double()
    log_q = torch.log_softmax(l, dim=1).gather(1, ids.clamp(min=0))
    kept = (ids != example.EMPTY) & torch.isfinite(log_q)
    cz = (example.SCALE * scores.double()).masked_fill(~kept, -1e300)
    log_p = torch.log_softmax(cz, dim=1)
    terms = torch.where(kept, log_p.exp() * (log_p - log_q.masked_fill(~kept, 0.0)), 0.0)
    want = terms.sum(dim=1).mean()
    want.backward()
    want = want.detach()
    # vectors are float32 sums of 24 terms, logits of 16 times 20: off by (24 + 16 / 16 + 4) 2^-23
    # times sums of magnitudes, at most some 4 times the largest logit of about 30; shares by twice
    # that, 2^-11 of themselves for the largest, and a gradient's norm by less than the worst share
    assert abs(float(loss) - float(want)) <= 2.0 ** -11
    for got, ref in ((dtable, table.grad), (dw, w.grad)):
        assert float((got.double() - ref).norm()) <= 2.0 ** -11 * float(ref.norm())


def test_the_run_in_one_graph(example):
    # a step's kernels captured once and replayed on new data give what calls give
    head = example.Head(300, 64, 32, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    items = torch.randn(3000, 32, generator=g, device="cuda")

    def batch():
        return (torch.randint(0, 300, (40, 5), generator=g, device="cuda"),
                torch.randint(0, 3000, (40, 12), generator=g, device="cuda"),
                torch.rand(40, 12, generator=g, device="cuda"))

    def call(tokens, ids, scores):
        loss, dtable, dw = head.gradients(tokens, items, ids, scores)
        packed = pvs.pvs_mx_pack(head.w, example.GROUP)
        return loss, dtable, dw, head.vectors(tokens, packed)

    kept = batch()
    call(*kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(*kept)
    for _ in range(3):
        new = batch()
        for a, b in zip(kept, new):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, call(*new)):
            assert torch.equal(a, b)


def test_calls_from_two_streams_at_once(example):
    # each call has its own scratch: calls in flight together do not meet
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(300, 256, generator=g, device="cuda").bfloat16()
    w = torch.randn(20_000, 256, generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, 20_000, (300, 16), generator=g, device="cuda")
    z = torch.randn(300, 16, generator=g, device="cuda")
    dy = torch.randn(20_000, 256, generator=g, device="cuda").bfloat16()
    token = torch.randint(0, 5000, (20_000,), generator=g, device="cuda")
    packed = pvs.pvs_mx_pack(w, 16)

    def work():
        return (*pvs.pvs_distill_forward(x, w, ids, z), pvs.pvs_embed_backward(dy, token, 5000),
                pvs.pvs_mx_matmul(x, *packed, 16))

    want = work()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(work())
    torch.cuda.synchronize()
    for out in got:
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_vectors_of_the_packed_layer(example):
    # serving: the rows' sums and the product of what both packed operands stand for, in binary64
    head = example.Head(200, 128, 64, seed=8)
    g = torch.Generator(device="cuda").manual_seed(9)
    tokens = torch.randint(0, 200, (300, 6), generator=g, device="cuda")
    tokens[torch.rand(300, 6, generator=g, device="cuda") < 0.2] = example.EMPTY
    tokens[:, 0] = torch.arange(300, device="cuda") % 200
    rows = head.table.double()[tokens.clamp(min=0)] * (tokens != example.EMPTY)[..., None]
    x = head.pooled(tokens)
    # six float32 products and their sum
    assert ((x.double() - rows.sum(dim=1) * 6 ** -0.5).abs() <= 6 * 2.0 ** -23 * rows.abs().sum(dim=1)).all()
    packed = pvs.pvs_mx_pack(head.w, example.GROUP)

    def stands_for(p):
        return pvs.pvs_mx_unpack(*p, example.GROUP, 128, torch.float32).double()

    want = stands_for(pvs.pvs_mx_pack(x, example.GROUP)) @ stands_for(packed).T
    want = want / want.norm(dim=1, keepdim=True)
    got = head.vectors(tokens, packed)
    # (128 / 64 + 8) 2^-23 of sums of magnitudes, which are about 0.64 128^1/2 = 7.2 times as large as the
    # sums: 72 2^-23, and some 2^-22 for the norm
    assert float((got.double() - want).norm(dim=1).max()) <= 2.0 ** -16
    # against the float32 layer: a code is off by a fifth of its element at most (from 5/2), by about a
    # tenth in the mean, in both operands and alike in no direction: 0.15 of a vector, a third of the bound
    exact = head.vectors(tokens).double()
    assert float((got.double() - exact).norm(dim=1).max()) <= 0.5
