"""The operators of a trained projection head, as cases that can be measured.

A head turns an encoder's hidden rows into the vectors that an index holds.  It is
trained with a softmax over the items of a collection, keeps its activations in
8 bits between the two passes, and is served with 4-bit weights.  Kinds:

* ``xent_loss``  cross entropy of T rows over V items, no gradient;
* ``xent_step``  the same with the gradients of both operands;
* ``ckpt_store`` rows kept in 8 bits (with their GELU where ``gelu``), and what they stand for;
* ``ckpt_grad``  a layer's backward pass from rows kept in 8 bits: the GELU's gradient
                 and the weight's;
* ``wq_matvec``  a few rows times 4-bit weights with group scales;
* ``wq_pack``    weights put into 4 bits, and what they stand for.

Rows and items are noisy unit vectors, as an index holds them; a row's target is
the item that it was drawn around.
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
        # one query's loss over a small collection: launches and latency
        dict(name="xent_loss_one", kind="xent_loss", T=1, V=10_000, d=128, dtype="bf16", masked=0.0, ignored=0.0),
        # a validation batch of an index width that fits no tile, deletions masked, float32 as the index takes it
        dict(name="xent_loss_ragged", kind="xent_loss", T=200, V=100_003, d=385, dtype="f32", masked=0.02, ignored=0.1),
        # in-batch negatives: every row's passage is every other row's negative
        dict(name="xent_step_inbatch", kind="xent_step", T=8192, V=8192, d=768, dtype="bf16", masked=0.0, ignored=0.0),
        # a query batch against a whole collection of a million passages
        dict(name="xent_step_1M", kind="xent_step", T=256, V=1_000_000, d=768, dtype="bf16", masked=0.02, ignored=0.0),
        # token-level training over a large vocabulary, f16 with a scaled loss
        dict(name="xent_step_200k", kind="xent_step", T=4096, V=200_000, d=1024, dtype="f16", masked=0.0, ignored=0.1),
        # float32 vectors of an odd width, deletions and ignored rows
        dict(name="xent_step_ragged", kind="xent_step", T=777, V=20_011, d=385, dtype="f32", masked=0.02, ignored=0.1),
        # the hidden rows of a head's first layer, kept in 8 bits with their GELU
        dict(name="ckpt_store_gelu", kind="ckpt_store", R=32_768, K=1536, dtype="bf16", gelu=True),
        # that layer's backward pass
        dict(name="ckpt_grad_layer", kind="ckpt_grad", R=32_768, N=1536, K=768, dtype="bf16"),
        # a small odd layer in float32
        dict(name="ckpt_grad_ragged", kind="ckpt_grad", R=1001, N=385, K=770, dtype="f32"),
        # one query through a served head
        dict(name="wq_matvec_head", kind="wq_matvec", B=1, N=768, K=768, group=64, dtype="bf16"),
        # a few queries scored against every item of a million, in 4 bits
        dict(name="wq_matvec_1M", kind="wq_matvec", B=4, N=1_000_000, K=768, group=128, dtype="f32"),
        # a collection's matrix put into 4 bits
        dict(name="wq_pack_200k", kind="wq_pack", N=200_000, K=1000, group=32, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["xent_loss", "xent_step", "xent_step", "ckpt_store", "ckpt_grad", "wq_matvec", "wq_matvec", "wq_pack"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("xent_loss", "xent_step"):
        d = rng.choice([64, 128, 384, 768, 1024, rng.randint(33, 1024)])
        T = _log(rng, 1, 8192)
        V = _log(rng, 100, 1_000_000)
        V = max(64, min(V, 200_000 * 4096 // T, 768_000_000 // d))
        return dict(kind=kind, T=T, V=V, d=d, dtype=dtype, masked=rng.choice([0.0, 0.02, 0.5]), ignored=rng.choice([0.0, 0.1]))
    if kind == "ckpt_store":
        K = _log(rng, 48, 8192)
        return dict(kind=kind, R=max(1, min(_log(rng, 1, 100_000), 50_000_000 // K)), K=K, dtype=dtype, gelu=rng.random() < 0.5)
    if kind == "ckpt_grad":
        N, K = _log(rng, 64, 4096), _log(rng, 64, 4096)
        return dict(kind=kind, R=max(1, min(_log(rng, 1, 65_536), 60_000_000 // max(N, K))), N=N, K=K, dtype=dtype)
    K = _log(rng, 32, 8192)
    N = max(1, min(_log(rng, 64, 1_000_000), 768_000_000 // K))
    group = rng.choice([32, 64, 128])
    if kind == "wq_pack":
        return dict(kind=kind, N=max(1, min(N, 200_000_000 // K)), K=K, group=group, dtype=dtype)
    return dict(kind=kind, B=rng.choice([1, 1, 2, 3, 4, 8, 16]), N=N, K=K, group=group, dtype=dtype)


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


def _stored_rows(x):
    """Scales and 8-bit codes of rows: s = max|x| / 127 in float32, codes rounded half away from zero."""
    top = x.abs().amax(dim=1, keepdim=True)
    s = torch.where(top > 0, top / 127.0, torch.ones_like(top))
    return s, _half_away(x / s).clamp(-127, 127)


def _half_away(q):
    whole = torch.trunc(q)
    return whole + torch.sign(q) * ((q - whole).abs() >= 0.5)


def _padded(k):
    return -(-k // 128) * 128


def _packed_weights(w, group):
    """float32 [N, K]: whole codes in [-7, 7] [N, padded K] and bf16 scales [N, padded K / group]."""
    n, k = w.shape
    w = torch.nn.functional.pad(w, (0, _padded(k) - k)).reshape(n, -1, group)
    top = w.abs().amax(dim=2)
    s = torch.where(top > 0, top / 7.0, torch.ones_like(top)).to(torch.bfloat16)
    return _half_away(w / s.float()[..., None]).clamp(-7, 7).reshape(n, -1), s


def _nibbles(q):
    """Codes [N, padded K] as bytes: in each block of 128, byte 16 t + 4 i + b holds k = 32 i + 8 t + 2 b and k + 1."""
    u = (q + 8).to(torch.uint8).reshape(q.shape[0], -1, 4, 4, 4, 2).transpose(2, 3)
    return (u[..., 0] | (u[..., 1] << 4)).reshape(q.shape[0], -1).contiguous()


def _from_nibbles(codes):
    c = codes.reshape(codes.shape[0], -1, 4, 4, 4)
    u = torch.stack((c & 15, c >> 4), dim=-1).transpose(2, 3)
    return u.reshape(codes.shape[0], -1).float() - 8.0


def prepare(case, seed):
    g = _generator(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind in ("xent_loss", "xent_step"):
        T, V, d = case["T"], case["V"], case["d"]
        w = torch.empty(V, d, dtype=dtype, device=DEVICE)
        for i in range(0, V, 1 << 18):
            w[i:i + (1 << 18)] = _unit_rows(min(1 << 18, V - i), d, g)
        y = torch.randint(0, V, (T,), generator=g, device=DEVICE)
        bias = None
        if case["masked"]:
            # deleted items, and the correction for items sampled unevenly
            bias = -0.5 * torch.rand(V, generator=g, device=DEVICE)
            bias[torch.rand(V, generator=g, device=DEVICE) < case["masked"]] = -math.inf
            bias[y] = -0.25
        # a row's own item stands out of the others by a little: 20 cos = ln V, losses near one
        noise = math.sqrt((20.0 / max(1.0, math.log(V))) ** 2 - 1.0)
        x = w[y].float() + noise * _unit_rows(T, d, g)
        x = (x / x.norm(dim=1, keepdim=True)).to(dtype)
        if case["ignored"]:
            y[torch.rand(T, generator=g, device=DEVICE) < case["ignored"]] = IGNORE
        # the mean over the batch with uneven row weights; f16 is trained with a scaled loss
        grad = (0.5 + torch.rand(T, generator=g, device=DEVICE)) / T
        if dtype == torch.float16:
            grad = grad * 65536.0
        return dict(kind=kind, x=x, w=w, y=y, bias=bias, grad=grad, scale=20.0)
    if kind == "ckpt_store":
        return dict(kind=kind, x=_hidden(case["R"], case["K"], g).to(dtype), gelu=case["gelu"])
    if kind == "ckpt_grad":
        R, N, K = case["R"], case["N"], case["K"]
        # the layer's input (its weight's gradient) and its output before the GELU
        s_in, z_in = _stored_rows(_hidden(R, K, g))
        s_pre, z_pre = _stored_rows(_hidden(R, N, g))
        dy = (torch.randn(R, N, generator=g, device=DEVICE) * 0.02).to(dtype)
        return dict(kind=kind, dy=dy, z_in=z_in.to(torch.int8), s_in=s_in.reshape(-1), z_pre=z_pre.to(torch.int8),
                    s_pre=s_pre.reshape(-1))
    w = (torch.randn(case["N"], case["K"], generator=g, device=DEVICE) * case["K"] ** -0.5).to(dtype)
    if kind == "wq_pack":
        return dict(kind=kind, w=w, group=case["group"])
    n = case["N"]
    codes = torch.empty(n, _padded(case["K"]) // 2, dtype=torch.uint8, device=DEVICE)
    scales = torch.empty(n, _padded(case["K"]) // case["group"], dtype=torch.bfloat16, device=DEVICE)
    for i in range(0, n, 1 << 16):
        q, s = _packed_weights(w[i:i + (1 << 16)].float(), case["group"])
        codes[i:i + (1 << 16)], scales[i:i + (1 << 16)] = _nibbles(q), s
    x = torch.randn(case["B"], case["K"], generator=g, device=DEVICE).to(dtype)
    return dict(kind=kind, x=x, codes=codes, scales=scales, group=case["group"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2608_07152_gb300 as pvs
    kind = s["kind"]
    if kind in ("xent_loss", "xent_step"):
        loss, stats = pvs.pvs_xent_forward(s["x"], s["w"], s["y"], bias=s["bias"], scale=s["scale"], ignore_index=IGNORE)
        if kind == "xent_loss":
            return dict(loss=loss)
        dx, dw = pvs.pvs_xent_backward(s["x"], s["w"], s["y"], stats, s["grad"], bias=s["bias"], scale=s["scale"],
                                       ignore_index=IGNORE)
        return dict(loss=loss, dx=dx, dw=dw)
    if kind == "ckpt_store":
        codes, scales, y = pvs.pvs_ckpt_store(s["x"], act=pvs.PVS_ACT_GELU if s["gelu"] else pvs.PVS_ACT_NONE)
        kept = pvs.pvs_ckpt_load(codes, scales, s["x"].dtype)
        return dict(kept=kept, y=y) if s["gelu"] else dict(kept=kept)
    if kind == "ckpt_grad":
        dpre = pvs.pvs_ckpt_act_backward(s["dy"], s["z_pre"], s["s_pre"], pvs.PVS_ACT_GELU)
        return dict(dpre=dpre, dw=pvs.pvs_ckpt_grad_weight(dpre, s["z_in"], s["s_in"]))
    if kind == "wq_pack":
        codes, scales = pvs.pvs_wq_pack(s["w"], s["group"])
        return dict(weights=pvs.pvs_wq_unpack(codes, scales, s["group"], s["w"].shape[1], s["w"].dtype))
    return dict(y=pvs.pvs_wq_matvec(s["x"], s["codes"], s["scales"], s["group"]))


def _gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _gelu_slope(x):
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


def _run_plain(s):
    kind = s["kind"]
    if kind in ("xent_loss", "xent_step"):
        x, w, y = s["x"].float(), s["w"].float(), s["y"]
        logits = (x @ w.T) * s["scale"]
        if s["bias"] is not None:
            logits += s["bias"]
        top = logits.amax(dim=1, keepdim=True)
        kept = y != IGNORE
        at = torch.where(kept, y, torch.zeros_like(y))[:, None]
        hit = torch.gather(logits, 1, at) - top
        p = logits.sub_(top).exp_()
        total = p.sum(dim=1, keepdim=True)
        loss = torch.where(kept, (torch.log(total) - hit)[:, 0], torch.zeros_like(hit[:, 0]))
        if kind == "xent_loss":
            return dict(loss=loss)
        p.div_(total)
        p.scatter_add_(1, at, torch.full_like(hit, -1.0))
        p.mul_(torch.where(kept, s["grad"] * s["scale"], torch.zeros_like(s["grad"]))[:, None])
        return dict(loss=loss, dx=(p @ w).to(s["x"].dtype), dw=(p.T @ x).to(s["w"].dtype))
    if kind == "ckpt_store":
        x = s["x"].float()
        scale, z = _stored_rows(x)
        kept = (z * scale).to(s["x"].dtype)
        return dict(kept=kept, y=_gelu(x).to(s["x"].dtype)) if s["gelu"] else dict(kept=kept)
    if kind == "ckpt_grad":
        dpre = s["dy"].float() * _gelu_slope(s["z_pre"].float() * s["s_pre"][:, None])
        dpre = dpre.to(s["dy"].dtype)
        dw = dpre.float().T @ (s["z_in"].float() * s["s_in"][:, None])
        return dict(dpre=dpre, dw=dw.to(s["dy"].dtype))
    if kind == "wq_pack":
        q, scale = _packed_weights(s["w"].float(), s["group"])
        weights = q * scale.float().repeat_interleave(s["group"], dim=1)
        return dict(weights=weights[:, :s["w"].shape[1]].to(s["w"].dtype))
    x = s["x"].float()
    w = _from_nibbles(s["codes"]) * s["scales"].float().repeat_interleave(s["group"], dim=1)
    return dict(y=(x @ w[:, :x.shape[1]].T).to(s["x"].dtype))


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    kind = case["kind"]
    if kind in ("xent_loss", "xent_step"):
        T, V, d = case["T"], case["V"], case["d"]
        operands = (T + V) * d * size
        if kind == "xent_loss":
            return {"bytes": operands + 12 * T, "flops": 2 * T * V * d}
        return {"bytes": 2 * operands + 16 * T, "flops": 6 * T * V * d}
    if kind == "ckpt_store":
        n = case["R"] * case["K"]
        return {"bytes": n * (2 * size + (size if case["gelu"] else 0)), "flops": 10 * n}
    if kind == "ckpt_grad":
        R, N, K = case["R"], case["N"], case["K"]
        return {"bytes": R * N * (2 * size + 1) + R * K + N * K * size + 8 * R, "flops": 2 * R * N * K + 20 * R * N}
    N, K = case["N"], _padded(case["K"])
    if kind == "wq_pack":
        return {"bytes": 2 * N * case["K"] * size, "flops": 5 * N * K}
    return {"bytes": N * K // 2 + 2 * N * K // case["group"] + case["B"] * (case["K"] + N) * size,
            "flops": 2 * case["B"] * N * case["K"]}


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind in ("xent_loss", "xent_step"):
        # a log-probability a piece of rows at a time, so that the logits fit in 64 bits
        w = s["w"].to(torch.float64)
        loss, dx, dw = [], [], torch.zeros_like(w)
        step = max(1, (1 << 29) // w.shape[0])
        for i in range(0, s["x"].shape[0], step):
            x, y = s["x"][i:i + step].to(torch.float64), s["y"][i:i + step]
            logp = s["scale"] * torch.mm(x, w.t())
            if s["bias"] is not None:
                logp = logp + s["bias"].to(torch.float64)
            logp = logp - torch.logsumexp(logp, dim=1, keepdim=True)
            kept = (y != IGNORE).to(torch.float64)
            rows, cols = torch.arange(y.numel(), device=y.device), y.clamp(min=0)
            loss.append(-logp[rows, cols] * kept)
            if kind == "xent_step":
                soft = logp.exp()
                soft[rows, cols] -= 1.0
                soft *= (kept * s["grad"][i:i + step].to(torch.float64) * s["scale"])[:, None]
                dx.append(torch.mm(soft, w))
                dw.addmm_(soft.t(), x)
        return dict(loss=torch.cat(loss)) if kind == "xent_loss" else dict(loss=torch.cat(loss), dx=torch.cat(dx), dw=dw)
    if kind == "ckpt_store":
        x = s["x"].to(torch.float64)
        peak = x.abs().max(dim=1, keepdim=True).values
        # the scale that is kept is a float32
        unit = torch.where(peak > 0, (peak / 127.0).to(torch.float32).to(torch.float64), torch.ones_like(peak))
        z = torch.sign(x) * torch.clamp(torch.floor(x.abs() / unit + 0.5), max=127.0)
        if not s["gelu"]:
            return dict(kept=unit * z)
        return dict(kept=unit * z, y=x * 0.5 * torch.erfc(-x / math.sqrt(2.0)))
    if kind == "ckpt_grad":
        pre = s["z_pre"].to(torch.float64) * s["s_pre"].to(torch.float64)[:, None]
        slope = 0.5 * torch.erfc(-pre / math.sqrt(2.0)) + pre * torch.exp(-pre.square() / 2) / math.sqrt(2 * math.pi)
        dpre = s["dy"].to(torch.float64) * slope
        rows = s["z_in"].to(torch.float64) * s["s_in"].to(torch.float64)[:, None]
        return dict(dpre=dpre, dw=torch.mm(dpre.t(), rows))
    if kind == "wq_pack":
        n, group = case["N"], s["group"]
        w = torch.zeros(n, _padded(case["K"]), dtype=torch.float64, device=DEVICE)
        w[:, :case["K"]] = s["w"]
        w = w.view(n, -1, group)
        peak = w.abs().max(dim=2, keepdim=True).values
        # the scale that is kept is a bf16, rounded from float32
        unit = torch.where(peak > 0, (peak / 7.0).float().bfloat16().to(torch.float64), torch.ones_like(peak))
        weights = unit * torch.sign(w) * torch.clamp(torch.floor(w.abs() / unit + 0.5), max=7.0)
        return dict(weights=weights.view(n, -1)[:, :case["K"]])
    y = torch.zeros(case["B"], case["N"], dtype=torch.float64, device=DEVICE)
    for k in range(case["K"]):
        at = (k // 128) * 64 + 16 * (k % 32 // 8) + 4 * (k % 128 // 32) + k % 8 // 2
        q = (s["codes"][:, at].to(torch.int16) >> (4 * (k % 2))) & 15
        weight = (q.to(torch.float64) - 8.0) * s["scales"][:, k // s["group"]].to(torch.float64)
        y += s["x"][:, k, None].to(torch.float64) * weight
    return dict(y=y)
