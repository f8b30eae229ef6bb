"""More operators of a trained projection head, as cases that can be measured.

What a head is fed with, what else it learns from, and how it encodes many rows at once.
Kinds:

* ``distill_loss`` T rows over V items against a teacher's K best logits of each row, no gradient;
* ``distill_step`` the same with the gradients of both operands;
* ``embed_lookup`` rows of a table, scaled;
* ``embed_step``   a lookup and the gradient of the table from the looked-up rows' gradient;
* ``mx_pack``      rows put into microscaled 4-bit floating point, and what they stand for;
* ``mx_matmul``    B rows, put into that format on the way, times weights kept in it.

Rows and items are noisy unit vectors, as an index holds them; a teacher's list starts with the
item that the row was drawn around.  Token ids follow Zipf's law.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda"
IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one query's list over a small collection: launches and latency
        dict(name="distill_loss_one", kind="distill_loss", T=1, V=10_000, d=128, K=32, dtype="bf16", masked=0.0, empty=0.0),
        # a validation batch of an index width that fits no tile, deletions masked, lists that are not full
        dict(name="distill_step_ragged", kind="distill_step", T=200, V=100_003, d=385, K=100, dtype="f32", masked=0.02, empty=0.1),
        # in-batch negatives with a reranker's scores of some of them
        dict(name="distill_step_inbatch", kind="distill_step", T=4096, V=8192, d=768, K=64, dtype="bf16", masked=0.0, empty=0.0),
        # token-level training over a large vocabulary, f16 with a scaled loss
        dict(name="distill_step_200k", kind="distill_step", T=2048, V=200_000, d=1024, K=128, dtype="f16", masked=0.0, empty=0.1),
        # one short query's tokens
        dict(name="embed_lookup_one", kind="embed_lookup", n=16, V=50_000, d=768, dtype="bf16", empty=0.0),
        # a batch of passages' tokens, forward and backward
        dict(name="embed_step_200k", kind="embed_step", n=131_072, V=200_000, d=1024, dtype="bf16", empty=0.1),
        # a small odd table in float32
        dict(name="embed_step_ragged", kind="embed_step", n=5000, V=10_007, d=385, dtype="f32", empty=0.1),
        # a collection's matrix put into 4 bits, with scales of powers of two
        dict(name="mx_pack_200k", kind="mx_pack", R=200_000, K=1000, group=32, dtype="f16"),
        # a layer's weights of an odd shape, with fine scales
        dict(name="mx_pack_ragged", kind="mx_pack", R=1537, K=771, group=16, dtype="f32"),
        # one query through a served head
        dict(name="mx_matmul_one", kind="mx_matmul", B=1, N=768, K=768, group=16, dtype="bf16"),
        # a few queries against every item of a million, in 4 bits
        dict(name="mx_matmul_1M", kind="mx_matmul", B=32, N=1_000_000, K=768, group=32, dtype="bf16"),
        # a wide layer over a corpus of passages
        dict(name="mx_matmul_corpus", kind="mx_matmul", B=16_384, N=4096, K=4096, group=16, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["distill_loss", "distill_step", "distill_step", "embed_lookup", "embed_step", "mx_pack", "mx_matmul", "mx_matmul"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("distill_loss", "distill_step"):
        d = rng.choice([64, 128, 384, 768, 1024, rng.randint(33, 1024)])
        T = _log(rng, 1, 8192)
        V = _log(rng, 100, 1_000_000)
        V = max(64, min(V, 200_000 * 2048 // T, 768_000_000 // d))
        return dict(kind=kind, T=T, V=V, d=d, K=_log(rng, 1, 256), dtype=dtype, masked=rng.choice([0.0, 0.02, 0.5]),
                    empty=rng.choice([0.0, 0.1]))
    if kind in ("embed_lookup", "embed_step"):
        d = rng.choice([64, 128, 384, 768, 1024, rng.randint(33, 2048)])
        n = min(_log(rng, 1, 262_144), 131_072 * 1024 // d)
        return dict(kind=kind, n=n, V=min(_log(rng, 100, 1_000_000), 200_000 * 1024 // d), d=d, dtype=dtype,
                    empty=rng.choice([0.0, 0.1]))
    K = _log(rng, 32, 8192)
    group = rng.choice([16, 32])
    if kind == "mx_pack":
        return dict(kind=kind, R=max(1, min(_log(rng, 1, 1_000_000), 200_000_000 // K)), K=K, group=group, dtype=dtype)
    N = max(1, min(_log(rng, 64, 1_000_000), 768_000_000 // K))
    B = _log(rng, 1, 16_384)
    B = max(1, min(B, 16_384 * 4096 * 4096 // (N * K), 134_000_000 // N))
    return dict(kind=kind, B=B, N=N, K=K, group=group, dtype=dtype)


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _unit_rows(n, d, g):
    x = torch.randn(n, d, generator=g, device=DEVICE)
    return x / x.norm(dim=1, keepdim=True)


def _hidden(r, k, g):
    # rows of unlike sizes with a few large channels, as hidden states have them
    size = torch.exp(0.5 * torch.randn(r, 1, generator=g, device=DEVICE))
    channel = torch.exp(0.7 * torch.randn(1, k, generator=g, device=DEVICE))
    return torch.randn(r, k, generator=g, device=DEVICE) * size * channel


def _padded(k):
    return -(-k // 128) * 128


# ---- microscaled rows ------------------------------------------------------------------
# Element values of the codes 0 to 7; bit 3 is the sign.
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(e):
    """2^e in float32, e whole numbers in [-149, 127], made from its bits."""
    normal = ((e.clamp(min=-126) + 127) << 23).to(torch.int32)
    below = torch.ones_like(normal) << (e + 149).clamp(0, 22).to(torch.int32)
    return torch.where(e >= -126, normal, below).view(torch.float32)


def _exponent(x):
    """floor(log2 x) of positive float32 numbers."""
    return (torch.frexp(x).exponent - 1).to(torch.int64)


def _encode(x, group):
    """float32 [R, K]: codes uint8 [R, padded K], scale bytes uint8 [R, padded K / group], row scales float32 [R] or
    None, and what an element's code is in units of [R, padded K / group]."""
    r, k = x.shape
    x = torch.nn.functional.pad(x, (0, _padded(k) - k)).reshape(r, -1, group)
    top = x.abs().amax(dim=2)
    if group == 32:
        e = torch.where(top > 0, (_exponent(top) - 2).clamp(min=-127), torch.full_like(top, -127, dtype=torch.int64))
        scales, rows, unit = (e + 127).to(torch.uint8), None, _power(e)
    else:
        most = top.amax(dim=1)
        rows = torch.where(most > 0, _power((_exponent(most) - 10).clamp(min=-126)), torch.ones_like(most))
        s = (top / 6.0 / rows[:, None]).to(torch.float8_e4m3fn)
        scales, unit = s.view(torch.uint8), s.float() * rows[:, None]
    # a multiple of half a unit has few digits: which side of a border an element lies on is seen exactly
    a, u = x.abs(), unit[..., None]
    code = (a > 0.25 * u).to(torch.uint8)
    code += a >= 0.75 * u
    code += a > 1.25 * u
    code += a >= 1.75 * u
    code += a > 2.5 * u
    code += a >= 3.5 * u
    code += a > 5.0 * u
    code = torch.where((x < 0) & (code > 0), code + 8, code) * (u > 0)
    return code.reshape(r, -1), scales, rows, unit


def _decode(code, unit):
    """What codes [R, padded K] stand for in units [R, padded K / group], float32."""
    levels = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), dtype=torch.float32, device=code.device)
    return (levels[code.long()].reshape(*unit.shape, -1) * unit[..., None]).reshape(code.shape)


def _blocked(scales, group):
    """Scale bytes [R, padded K / group] as [ceil(R / 128), padded K / (4 group), 512]: a block holds four scales of 128
    rows, those of row 32 i + j at byte 16 j + 4 i."""
    r, n = scales.shape
    s = torch.nn.functional.pad(scales, (0, 0, 0, -r % 128)).reshape(-1, 4, 32, n // 4, 4)
    return s.permute(0, 3, 2, 1, 4).reshape(s.shape[0], n // 4, 512).contiguous()


def _rows_of_blocks(blocks, r):
    s = blocks.reshape(blocks.shape[0], blocks.shape[1], 32, 4, 4).permute(0, 3, 2, 1, 4)
    return s.reshape(blocks.shape[0] * 128, -1)[:r]


def _unit_of(scales, rows, group):
    if group == 32:
        return _power(scales.to(torch.int64) - 127)
    return scales.view(torch.float8_e4m3fn).float() * rows[:, None]


def _packed(x, group):
    code, scales, rows, _ = _encode(x, group)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales, rows


def _unpacked(codes):
    return torch.stack((codes & 15, codes >> 4), dim=-1).reshape(codes.shape[0], -1)


# ---- states ----------------------------------------------------------------------------
def prepare(case, seed):
    g = _generator(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind in ("distill_loss", "distill_step"):
        T, V, d, K = case["T"], case["V"], case["d"], case["K"]
        w = torch.empty(V, d, dtype=dtype, device=DEVICE)
        for i in range(0, V, 1 << 18):
            w[i:i + (1 << 18)] = _unit_rows(min(1 << 18, V - i), d, g)
        ids = torch.randint(0, V, (T, K), generator=g, device=DEVICE)
        bias = None
        if case["masked"]:
            # deleted items (some are in a list that is older than their deletion), and the correction for items
            # sampled unevenly
            bias = -0.5 * torch.rand(V, generator=g, device=DEVICE)
            bias[torch.rand(V, generator=g, device=DEVICE) < case["masked"]] = -math.inf
            bias[ids[:, 0]] = -0.25
        # a row's own item stands out of the others by a little: 20 cos = ln V, losses near one
        noise = math.sqrt((20.0 / max(1.0, math.log(V))) ** 2 - 1.0)
        x = w[ids[:, 0]].float() + noise * _unit_rows(T, d, g)
        x = (x / x.norm(dim=1, keepdim=True)).to(dtype)
        # a reranker's scores, best first
        z = (2.0 * torch.randn(T, K, generator=g, device=DEVICE)).sort(dim=1, descending=True).values
        z[:, 0] += 2.0
        if case["empty"]:
            # short lists, and rows without one
            short = torch.rand(T, K, generator=g, device=DEVICE) < case["empty"]
            short[:, 0] = False
            ids[short] = IGNORE
            ids[torch.rand(T, generator=g, device=DEVICE) < case["empty"]] = IGNORE
        # the mean over the batch with uneven row weights; f16 is trained with a scaled loss
        grad = (0.5 + torch.rand(T, generator=g, device=DEVICE)) / T
        if dtype == torch.float16:
            grad = grad * 65536.0
        return dict(kind=kind, x=x, w=w, ids=ids, z=z, bias=bias, grad=grad, scale=20.0, teacher_scale=0.8)
    if kind in ("embed_lookup", "embed_step"):
        n, V, d = case["n"], case["V"], case["d"]
        w = (0.02 * torch.randn(V, d, generator=g, device=DEVICE)).to(dtype)
        # frequent tokens first, a token's share falling as 1 / rank
        ids = torch.exp(torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64) * math.log(V)).long().clamp(max=V) - 1
        if case["empty"]:
            ids[torch.rand(n, generator=g, device=DEVICE) < case["empty"]] = IGNORE
        dy = (torch.randn(n, d, generator=g, device=DEVICE) * 0.01).to(dtype)
        return dict(kind=kind, w=w, ids=ids, dy=dy, scale=math.sqrt(d))
    if kind == "mx_pack":
        return dict(kind=kind, x=_hidden(case["R"], case["K"], g).to(dtype), group=case["group"])
    n, k, group = case["N"], case["K"], case["group"]
    codes = torch.empty(n, _padded(k) // 2, dtype=torch.uint8, device=DEVICE)
    scales = torch.empty(n, _padded(k) // group, dtype=torch.uint8, device=DEVICE)
    rows = torch.empty(n, device=DEVICE) if group == 16 else None
    for i in range(0, n, 1 << 16):
        w = torch.randn(min(1 << 16, n - i), k, generator=g, device=DEVICE) * k ** -0.5
        codes[i:i + (1 << 16)], scales[i:i + (1 << 16)], r = _packed(w.to(torch.bfloat16).float(), group)
        if rows is not None:
            rows[i:i + (1 << 16)] = r
    x = _hidden(case["B"], k, g).to(dtype)
    return dict(kind=kind, x=x, codes=codes, scales=_blocked(scales, group), rows=rows, group=group)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2608_07152_gb300 as pvs
    kind = s["kind"]
    if kind in ("distill_loss", "distill_step"):
        loss, stats, hits = pvs.pvs_distill_forward(s["x"], s["w"], s["ids"], s["z"], bias=s["bias"], scale=s["scale"],
                                                    teacher_scale=s["teacher_scale"], ignore_index=IGNORE)
        if kind == "distill_loss":
            return dict(loss=loss)
        dx, dw = pvs.pvs_distill_backward(s["x"], s["w"], s["ids"], stats, hits, s["grad"], bias=s["bias"], scale=s["scale"],
                                          ignore_index=IGNORE)
        return dict(loss=loss, dx=dx, dw=dw)
    if kind == "embed_lookup":
        return dict(y=pvs.pvs_embed_forward(s["w"], s["ids"], scale=s["scale"], ignore_index=IGNORE))
    if kind == "embed_step":
        y = pvs.pvs_embed_forward(s["w"], s["ids"], scale=s["scale"], ignore_index=IGNORE)
        dw = pvs.pvs_embed_backward(s["dy"], s["ids"], s["w"].shape[0], scale=s["scale"], ignore_index=IGNORE)
        return dict(y=y, dw=dw)
    if kind == "mx_pack":
        codes, scales, rows = pvs.pvs_mx_pack(s["x"], s["group"])
        return dict(values=pvs.pvs_mx_unpack(codes, scales, rows, s["group"], s["x"].shape[1], torch.float32))
    return dict(y=pvs.pvs_mx_matmul(s["x"], s["codes"], s["scales"], s["rows"], s["group"]))


def _run_plain(s):
    kind = s["kind"]
    if kind in ("distill_loss", "distill_step"):
        x, w = s["x"].float(), s["w"].float()
        logits = (x @ w.T) * s["scale"]
        if s["bias"] is not None:
            logits += s["bias"]
        kept = s["ids"] != IGNORE
        at = torch.where(kept, s["ids"], torch.zeros_like(s["ids"]))
        hit = torch.gather(logits, 1, at)
        # items that were deleted leave the list
        kept &= hit > -math.inf
        z = torch.where(kept, s["z"].float() * s["teacher_scale"], torch.full_like(hit, -math.inf))
        some = kept.any(dim=1, keepdim=True)
        z = z - torch.where(some, z.amax(dim=1, keepdim=True), torch.zeros_like(hit[:, :1]))
        e = torch.exp(z)
        share = e.sum(dim=1, keepdim=True)
        share = torch.where(some, share, torch.ones_like(share))
        teacher, log_teacher = e / share, z - torch.log(share)
        top = logits.amax(dim=1, keepdim=True)
        hit = hit - top
        p = logits.sub_(top).exp_()
        total = p.sum(dim=1, keepdim=True)
        terms = teacher * (log_teacher - hit + torch.log(total))
        loss = torch.where(kept, terms, torch.zeros_like(terms)).sum(dim=1)
        if kind == "distill_loss":
            return dict(loss=loss)
        p.div_(total)
        p.scatter_add_(1, at, -teacher)
        p.mul_(torch.where(some[:, 0], s["grad"] * s["scale"], torch.zeros_like(s["grad"]))[:, None])
        return dict(loss=loss, dx=(p @ w).to(s["x"].dtype), dw=(p.T @ x).to(s["w"].dtype))
    if kind in ("embed_lookup", "embed_step"):
        kept = s["ids"] != IGNORE
        at = torch.where(kept, s["ids"], torch.zeros_like(s["ids"]))
        rows = s["w"][at].float() * s["scale"]
        y = torch.where(kept[:, None], rows, torch.zeros_like(rows)).to(s["w"].dtype)
        if kind == "embed_lookup":
            return dict(y=y)
        dy = torch.where(kept[:, None], s["dy"].float() * s["scale"], torch.zeros_like(rows))
        dw = torch.zeros(s["w"].shape, dtype=torch.float32, device=dy.device).index_add_(0, at, dy)
        return dict(y=y, dw=dw.to(s["w"].dtype))
    if kind == "mx_pack":
        code, _, _, unit = _encode(s["x"].float(), s["group"])
        return dict(values=_decode(code, unit)[:, :s["x"].shape[1]])
    n = s["codes"].shape[0]
    w = _decode(_unpacked(s["codes"]), _unit_of(_rows_of_blocks(s["scales"], n), s["rows"], s["group"]))
    code, _, _, unit = _encode(s["x"].float(), s["group"])
    return dict(y=(_decode(code, unit) @ w.T).to(s["x"].dtype))


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    kind = case["kind"]
    if kind in ("distill_loss", "distill_step"):
        T, V, d, K = case["T"], case["V"], case["d"], case["K"]
        operands = (T + V) * d * size
        if kind == "distill_loss":
            return {"bytes": operands + 12 * T * K + 4 * T, "flops": 2 * T * V * d}
        return {"bytes": 2 * operands + 12 * T * K + 8 * T, "flops": 6 * T * V * d}
    if kind in ("embed_lookup", "embed_step"):
        n, V, d = case["n"], case["V"], case["d"]
        # the rows of the table that are looked up: each once
        used = min(n, V)
        if kind == "embed_lookup":
            return {"bytes": (n + used) * d * size + 8 * n, "flops": n * d}
        return {"bytes": (2 * n + used + V) * d * size + 8 * n, "flops": 3 * n * d}
    K = _padded(case["K"])
    if kind == "mx_pack":
        n = case["R"] * case["K"]
        return {"bytes": n * (size + 4), "flops": 4 * n}
    B, N = case["B"], case["N"]
    return {"bytes": N * K // 2 + N * K // case["group"] + B * (case["K"] + N) * size, "flops": 2 * B * N * K}


# ---- the definitions in 64 bits --------------------------------------------------------
def _two(e):
    """2^e in 64 bits, e whole numbers, from its bits (a power function may miss it by a last digit)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_rows(x, group):
    """What microscaled rows stand for, [R, K] in 64 bits."""
    r, k = x.shape
    full = torch.zeros(r, _padded(k), dtype=torch.float64, device=x.device)
    full[:, :k] = x
    full = full.view(r, -1, group)
    peak = full.abs().max(dim=2, keepdim=True).values

    def binade(v):
        return torch.frexp(torch.where(v > 0, v, torch.ones_like(v))).exponent.to(torch.float64) - 1.0

    if group == 32:
        unit = _two((binade(peak) - 2.0).clamp(min=-127.0))
    else:
        most = peak.max(dim=1, keepdim=True).values
        row = _two((binade(most) - 10.0).clamp(min=-126.0))
        fine = (peak / (6.0 * row)).float().to(torch.float64)
        step = _two(binade(fine).clamp(min=-6.0) - 3.0)
        unit = torch.round(fine / step) * step * row
    q = torch.where(unit > 0, full / torch.where(unit > 0, unit, torch.ones_like(unit)), torch.zeros_like(full))
    step = _two(binade(q.abs()).clamp(min=0.0) - 1.0)
    q = (torch.round(q / step) * step).clamp(-6.0, 6.0)
    return (q * unit).view(r, -1)[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind in ("distill_loss", "distill_step"):
        # log-probabilities a piece of rows at a time, so that the logits fit in 64 bits
        w = s["w"].to(torch.float64)
        loss, dx, dw = [], [], torch.zeros_like(w)
        step = max(1, (1 << 29) // w.shape[0])
        for i in range(0, s["x"].shape[0], step):
            x, ids, z = s["x"][i:i + step].to(torch.float64), s["ids"][i:i + step], s["z"][i:i + step].to(torch.float64)
            logq = s["scale"] * torch.mm(x, w.t())
            if s["bias"] is not None:
                logq = logq + s["bias"].to(torch.float64)
            logq = logq - torch.logsumexp(logq, dim=1, keepdim=True)
            at = ids.clamp(min=0)
            mine = logq.gather(1, at)
            out = (ids < 0) | torch.isinf(mine)
            weight = torch.softmax((s["teacher_scale"] * z).masked_fill(out, -1e30), dim=1).masked_fill(out, 0.0)
            has = (~out).any(dim=1).to(torch.float64)
            mine = mine.masked_fill(out, 0.0)
            loss.append((torch.special.xlogy(weight, weight) - weight * mine).sum(dim=1))
            if kind == "distill_step":
                soft = logq.exp().scatter_add(1, at, -weight)
                soft *= (has * s["grad"][i:i + step].to(torch.float64) * s["scale"])[:, None]
                dx.append(torch.mm(soft, w))
                dw.addmm_(soft.t(), x)
        return dict(loss=torch.cat(loss)) if kind == "distill_loss" else dict(loss=torch.cat(loss), dx=torch.cat(dx), dw=dw)
    if kind in ("embed_lookup", "embed_step"):
        w, ids = s["w"].to(torch.float64), s["ids"]
        live = torch.nonzero(ids >= 0)[:, 0]
        y = torch.zeros(ids.shape[0], w.shape[1], dtype=torch.float64, device=w.device)
        y[live] = s["scale"] * w.index_select(0, ids[live])
        if kind == "embed_lookup":
            return dict(y=y)
        dw = torch.zeros_like(w).index_put_((ids[live],), s["scale"] * s["dy"][live].to(torch.float64), accumulate=True)
        return dict(y=y, dw=dw)
    if kind == "mx_pack":
        return dict(values=_exact_rows(s["x"].to(torch.float64), s["group"]))
    rows = _exact_rows(s["x"].to(torch.float64), s["group"])
    y = torch.zeros(case["B"], case["N"], dtype=torch.float64, device=DEVICE)
    level = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, 8.0, 12.0], dtype=torch.float64, device=DEVICE)
    group, step = s["group"], 1 << 15
    for i in range(0, case["N"], step):
        c = s["codes"][i:i + step].to(torch.int64)
        c = torch.stack((c % 16, c // 16), dim=2).view(c.shape[0], -1)
        w = 0.5 * level[c % 8] * (1.0 - 2.0 * (c // 8))
        r = torch.arange(i, i + c.shape[0], device=DEVICE)[:, None]
        j = torch.arange(c.shape[1] // group, device=DEVICE)[None, :]
        byte = s["scales"][r // 128, j // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + j % 4].to(torch.float64)
        if group == 32:
            unit = _two(byte - 127.0)
        else:
            e, m = torch.floor(byte / 8.0), byte % 8.0
            unit = torch.where(e > 0, (8.0 + m) * _two(e - 10.0), m * 2.0 ** -9) * s["rows"][i:i + step, None].to(torch.float64)
        w = (w.view(c.shape[0], -1, group) * unit[..., None]).view(c.shape[0], -1)[:, :case["K"]]
        y[:, i:i + step] = torch.mm(rows, w.t())
    return dict(y=y)
