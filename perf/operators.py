"""Performance cases of the operators around the expert layer in a training step, with their plain forms.

  router       gates of replayed expert ids from the router's logits, the balance loss over per-expert counts
               ("fwd"), and the logits' gradient ("bwd")
  block_norm   x' = res_scale * x + gate * RMSNorm(y; w_post), n = RMSNorm(x'; w_pre): the norms after one block and
               before the next with the residual stream between them ("fwd"), and all gradients ("bwd")
  orthogonal   momentum and five Newton-Schulz steps on every expert's weight gradient: the update of the
               Muon optimiser

A case is a dict of sizes and switches; `prepare` draws its inputs, `run` takes them through the operator: in plain
torch operations, or, with `own`, through the library.  `exact` is the definition in double precision.
"""
import math

import torch

own = False

DEV = "cuda"
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315


def listed():
    return [
        # one new token through the router of 128 experts: latency of the call is all there is
        dict(name="router_fwd_token", op="router", dir="fwd", n_mb=1, T=1, E=128, k=8, score="softmax", normalize=True, type="fp32",
             padded=0.0, masked=0.0),
        # sizes that divide nothing, padded sequences, experts masked out by group-limited routing, sigmoid scores
        dict(name="router_fwd_ragged", op="router", dir="fwd", n_mb=3, T=777, E=60, k=6, score="sigmoid", normalize=True, type="bf16",
             padded=0.2, masked=0.3),
        # a whole batch of long micro-batches (Qwen3-235B-A22B-shaped layer)
        dict(name="router_fwd_batch", op="router", dir="fwd", n_mb=32, T=16384, E=128, k=8, score="softmax", normalize=True, type="bf16",
             padded=0.1, masked=0.0),
        # its backward pass: gradients of gates and of the loss to the logits
        dict(name="router_bwd_batch", op="router", dir="bwd", n_mb=32, T=16384, E=128, k=8, score="softmax", normalize=True, type="bf16",
             padded=0.1, masked=0.0),
        # DeepSeek-V3-shaped: 256 sigmoid-scored experts, logits in fp32, experts masked out
        dict(name="router_bwd_sigmoid", op="router", dir="bwd", n_mb=8, T=4096, E=256, k=8, score="sigmoid", normalize=True, type="fp32",
             padded=0.0, masked=0.5),
        # one new token between two blocks
        dict(name="norm_fwd_token", op="block_norm", dir="fwd", T=1, h=4096, type="bf16", post=True, pre=True, gate="none"),
        # a long micro-batch, norms on both sides, one gate a token
        dict(name="norm_fwd_long", op="block_norm", dir="fwd", T=16384, h=4096, type="bf16", post=True, pre=True, gate="token"),
        # its backward pass
        dict(name="norm_bwd_long", op="block_norm", dir="bwd", T=16384, h=4096, type="bf16", post=True, pre=True, gate="token"),
        # an odd number of wide rows, residual stream in fp32, a gate for every element
        dict(name="norm_bwd_ragged", op="block_norm", dir="bwd", T=777, h=7168, type="fp32", post=True, pre=True, gate="element"),
        # the smallest experts: launches and short chains of dependent products
        dict(name="ortho_tiny", op="orthogonal", blocks=8, rows=128, cols=256, type="fp32", momentum=True, nesterov=True, rank=0),
        # odd sizes, tall matrices, gradients in bf16 of experts that saw few tokens (low rank), no momentum yet
        dict(name="ortho_ragged", op="orthogonal", blocks=5, rows=1001, cols=333, type="bf16", momentum=False, nesterov=False, rank=24),
        # gate projections of 32 of a Qwen3-235B-A22B-shaped layer's experts (one rank's share of several)
        dict(name="ortho_large", op="orthogonal", blocks=32, rows=1536, cols=4096, type="fp32", momentum=True, nesterov=True, rank=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("router", "block_norm", "orthogonal"))
    if op == "router":
        while True:
            E = _log_int(rng, 4, 1024)
            c = dict(op=op, dir=rng.choice(("fwd", "bwd")), n_mb=_log_int(rng, 1, 32), T=_log_int(rng, 1, 16384), E=E,
                     k=rng.randint(1, min(E // 2, 16)), score=rng.choice(("softmax", "sigmoid")), normalize=rng.random() < 0.7,
                     type=rng.choice(("bf16", "fp32")), padded=rng.choice((0.0, 0.1, 0.5)), masked=rng.choice((0.0, 0.0, 0.4)))
            if c["n_mb"] * c["T"] * (c["E"] + 4 * c["k"]) <= 32 * 16384 * 128:
                return c
    if op == "block_norm":
        while True:
            c = dict(op=op, dir=rng.choice(("fwd", "bwd")), T=_log_int(rng, 1, 16384), h=8 * _log_int(rng, 8, 1024), type=rng.choice(("bf16", "fp32")),
                     post=rng.random() < 0.7, pre=rng.random() < 0.8, gate=rng.choice(("none", "token", "element")))
            if c["T"] * c["h"] <= 8192 * 4096:
                return c
    while True:
        c = dict(op=op, blocks=_log_int(rng, 1, 64), rows=_log_int(rng, 16, 4096), cols=_log_int(rng, 16, 4096), type=rng.choice(("fp32", "bf16")),
                 momentum=rng.random() < 0.6, nesterov=rng.random() < 0.5, rank=rng.choice((0, 0, 0, 16)))
        if work(c)["flops"] <= 4e12:
            return c


def work(case):
    if case["op"] == "router":
        tok, E, k = case["n_mb"] * case["T"], case["E"], case["k"]
        size = 4 if case["type"] == "fp32" else 2
        byt = tok * (E * size + 4 * k + 1)
        if case["dir"] == "fwd":
            return dict(bytes=byt + 4 * tok * k + 8 * case["n_mb"] * E, flops=8 * tok * E)
        return dict(bytes=byt + 4 * tok * k + tok * E * size + 4 * case["n_mb"] * E, flops=12 * tok * E)
    if case["op"] == "block_norm":
        n, stream = case["T"] * case["h"], 4 if case["type"] == "fp32" else 2
        gate = dict(none=0, token=4 * case["T"], element=2 * n)[case["gate"]]
        if case["dir"] == "fwd":
            return dict(bytes=n * (2 * stream + 2 + 2 * case["pre"]) + gate + 4 * case["h"], flops=10 * n)
        # reads x', dx', y, dn and the gate; writes dx, dy and the gate's gradient
        return dict(bytes=n * (2 * stream + stream * case["pre"] + 2 * (case["post"] or case["gate"] != "none") + 2 * case["pre"] + 2) + 2 * gate + 12 * case["h"],
                    flops=24 * n)
    m, n = sorted((case["rows"], case["cols"]))
    size = 4 if case["type"] == "fp32" else 2
    # symmetric products are half a product
    return dict(bytes=case["blocks"] * m * n * (size + 2 + 8 * case["momentum"]),
                flops=case["blocks"] * 5 * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n))


# ---------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def prepare(case, seed):
    gen = _gen(seed)
    stream = torch.float32 if case["type"] == "fp32" else torch.bfloat16
    s = dict(case=case, buffers={})
    if case["op"] == "router":
        n_mb, T, E, k = case["n_mb"], case["T"], case["E"], case["k"]
        z = 1.5 * _randn(gen, n_mb, T, E) - torch.log(torch.arange(1, E + 1, device=DEV))[torch.randperm(E, generator=gen, device=DEV)]
        if case["masked"]:                                   # whole groups of experts are out of a token's reach
            groups = torch.rand((n_mb, T, 4), generator=gen, device=DEV)
            out = (groups < case["masked"]) & (groups > groups.amin(2, keepdim=True)) & (groups < groups.amax(2, keepdim=True))
            z.masked_fill_(out[..., torch.arange(E, device=DEV) * 4 // E], -math.inf)
        s["logits"] = z.to(stream)
        # the ids are replayed: the rollout's logits were not quite these
        s["ids"] = torch.topk(z + 0.1 * _randn(gen, n_mb, T, E), k, dim=2).indices.to(torch.int32)
        lengths = T - (torch.rand(n_mb, generator=gen, device=DEV) * 2 * case["padded"] * T).long()
        s["valid"] = (torch.arange(T, device=DEV)[None, :] < lengths[:, None]).to(torch.uint8) if case["padded"] else None
        s["scale"], s["coef"] = (2.5, 1e-2) if case["score"] == "sigmoid" else (1.0, 1e-2)
        if case["dir"] == "bwd":
            s["dgates"] = _randn(gen, n_mb, T, k)
            # gradients accumulate over the batch: each micro-batch's loss counts for its share
            s["dloss"] = torch.full((n_mb,), 4096.0, device=DEV)
            valid = torch.ones((n_mb, T), device=DEV) if s["valid"] is None else s["valid"].float()
            s["n_valid"] = valid.sum(1).to(torch.int32)
            counts = torch.zeros((n_mb, E), device=DEV)
            counts.scatter_add_(1, s["ids"].long().view(n_mb, -1), valid[..., None].expand(n_mb, T, k).reshape(n_mb, -1))
            s["counts"] = counts.to(torch.int32)
    elif case["op"] == "block_norm":
        T, h = case["T"], case["h"]
        s["y"] = (0.5 * _randn(gen, T, h) * torch.exp(0.5 * _randn(gen, T, 1))).to(torch.bfloat16)
        x = _randn(gen, T, h) * torch.exp(0.3 * _randn(gen, 1, h))
        s["w_post"] = (1 + 0.2 * _randn(gen, h)).to(torch.bfloat16) if case["post"] else None
        s["w_pre"] = (1 + 0.2 * _randn(gen, h)).to(torch.bfloat16) if case["pre"] else None
        s["gate"] = None if case["gate"] == "none" else (torch.sigmoid(_randn(gen, T)) if case["gate"] == "token"
                                                         else torch.sigmoid(_randn(gen, T, h)).to(torch.bfloat16))
        s["res_scale"], s["eps"] = 0.9, 1e-6
        s["x"] = x.to(stream)                                # backward: the stream behind the block, as the forward pass left it
        if case["dir"] == "bwd":
            s["dx_out"] = _randn(gen, T, h).to(stream)
            s["dn"] = _randn(gen, T, h).to(torch.bfloat16) if case["pre"] else None
    else:
        b, r, c = case["blocks"], case["rows"], case["cols"]
        if case["rank"]:                                     # an expert that saw few tokens
            g = torch.bmm(_randn(gen, b, r, case["rank"]), _randn(gen, b, case["rank"], c))
        else:                                                # many tokens: rows of unlike size
            g = _randn(gen, b, r, c) * torch.exp(0.5 * _randn(gen, b, r, 1))
        s["grad"] = (1e-3 * g).to(stream)
        s["momentum"] = 5e-3 * _randn(gen, b, r, c) if case["momentum"] else None
        s["mu"], s["scale"] = 0.95, 0.2 * math.sqrt(max(r, c))
    return s


# ---------------------------------------------------------------------------------------------
def _scores(z, score):
    """Log scores u; a masked expert's is -inf in either form."""
    return z if score == "softmax" else torch.clamp(z, max=0.0) - torch.log1p(torch.exp(-torch.abs(z)))


def _softmax(u):
    top = u.amax(-1, keepdim=True)
    e = torch.exp(u - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total))


def _router_plain(s, dtype):
    """The definition in `dtype`: gates, counts, n_valid, prob_mean, loss, or the logits' gradient."""
    c = s["case"]
    E, k = c["E"], c["k"]
    z, ids = s["logits"].to(dtype), s["ids"].long()
    valid = torch.ones(z.shape[:2], dtype=dtype, device=z.device) if s["valid"] is None else s["valid"].to(dtype)
    u = _scores(z, c["score"])
    p = _softmax(u)
    us = torch.gather(u, 2, ids)
    if c["normalize"]:
        part = _softmax(us)                                  # over the selected experts only
    elif c["score"] == "softmax":
        part = torch.gather(p, 2, ids)
    else:
        part = torch.exp(us)
    if c["dir"] == "fwd":
        counts = torch.zeros((c["n_mb"], E), dtype=torch.int64, device=z.device)
        for j in range(k):
            counts += ((ids[:, :, j, None] == torch.arange(E, device=z.device)) & (valid > 0)[..., None]).sum(1)
        n_valid = valid.double().sum(1)
        n = torch.clamp(n_valid, min=1.0)[:, None]
        mean = (p.double() * valid[..., None].double()).sum(1) / n
        loss = s["coef"] * E * (counts / (k * n) * mean).sum(1)
        return s["scale"] * part * valid[..., None], counts.to(torch.int32), n_valid.to(torch.int32), mean.to(dtype), loss.to(dtype)
    n = torch.clamp(s["n_valid"].to(dtype), min=1.0)[:, None]
    share = (s["dloss"].to(dtype)[:, None] * s["coef"] * E / k) * s["counts"].to(dtype) / (n * n)
    d = share[:, None, :].expand_as(z).clone()
    dg = s["scale"] * s["dgates"].to(dtype)
    if not c["normalize"] and c["score"] == "softmax":
        d.scatter_add_(2, ids, dg)
    du = p * (d - (d * p).sum(-1, keepdim=True))
    if c["normalize"]:
        du.scatter_add_(2, ids, part * (dg - (part * dg).sum(-1, keepdim=True)))
    elif c["score"] == "sigmoid":
        du.scatter_add_(2, ids, part * dg)
    if c["score"] == "sigmoid":
        du = du / (1 + torch.exp(z))
    return du * valid[..., None]


def _norm_plain(s, dtype):
    """The definition in `dtype`: (x', n) or (dx, dy, dgate, dw_post, dw_pre), absent ones left out."""
    c = s["case"]
    f = lambda name: None if s[name] is None else s[name].to(dtype)
    y, w2, w1 = f("y"), f("w_post"), f("w_pre")
    gate = f("gate")
    if gate is not None and gate.dim() == 1:
        gate = gate[:, None]
    r2 = 1 / torch.sqrt((y * y).mean(1, keepdim=True) + s["eps"])
    yh = y * r2
    z = y if w2 is None else yh * w2
    x = f("x")
    if c["dir"] == "fwd":
        x_out = s["res_scale"] * x + (z if gate is None else gate * z)
        if w1 is None:
            return (x_out,)
        r1 = 1 / torch.sqrt((x_out * x_out).mean(1, keepdim=True) + s["eps"])
        return x_out, x_out * r1 * w1
    D = f("dx_out")
    dw1 = None
    if w1 is not None:
        r1 = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + s["eps"])
        xh, dn = x * r1, f("dn")
        dw1 = (dn * xh).sum(0)
        D = D + r1 * (w1 * dn - xh * (w1 * dn * xh).mean(1, keepdim=True))
    dz = D if gate is None else gate * D
    dw2, dy = None, dz
    if w2 is not None:
        dw2 = (dz * yh).sum(0)
        dy = r2 * (dz * w2 - yh * (dz * w2 * yh).mean(1, keepdim=True))
    dgate = None
    if gate is not None:
        dgate = D * z
        if c["gate"] == "token":
            dgate = dgate.sum(1)
    return s["res_scale"] * D, dy, dgate, dw2, dw1


def _ortho_plain(s, dtype):
    c = s["case"]
    g = s["grad"].to(dtype)
    mom, u = None, g
    if s["momentum"] is not None:
        mom = s["mu"] * s["momentum"].to(dtype) + g
        u = g + s["mu"] * mom if c["nesterov"] else mom
    tall = c["rows"] > c["cols"]
    x = u.transpose(1, 2).contiguous() if tall else u
    norm = torch.sqrt((x.double() * x.double()).sum((1, 2), keepdim=True)).to(dtype)
    x = x / torch.where(norm > 0, norm, torch.ones_like(norm))
    for _ in range(5):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = NS_A * x + torch.bmm(NS_B * a + NS_C * torch.bmm(a, a), x)
    out = s["scale"] * x
    return out.transpose(1, 2).contiguous() if tall else out, mom


def _rounded(s, outs):
    """Each result in the type the operator gives it in."""
    c = s["case"]
    stream = torch.float32 if c["type"] == "fp32" else torch.bfloat16
    if c["op"] == "router":
        return outs if c["dir"] == "fwd" else (outs.to(stream),)
    if c["op"] == "block_norm":
        if c["dir"] == "fwd":
            types = (stream, torch.bfloat16)
        else:
            types = (stream, torch.bfloat16, torch.float32 if c["gate"] == "token" else torch.bfloat16, torch.float32, torch.float32)
    else:
        types = (torch.bfloat16, torch.float32)
    return tuple(o.to(t) for o, t in zip(outs, types) if o is not None)


def run(state):
    if own:
        return _run_own(state)
    plain = dict(router=_router_plain, block_norm=_norm_plain, orthogonal=_ortho_plain)[state["case"]["op"]]
    return _rounded(state, plain(state, torch.float32))


def _run_own(s):
    """The calls of a program that keeps its output buffers and workspaces from step to step."""
    import paper_2605_08639_amd as rl

    c, b = s["case"], s["buffers"]
    if not b:
        b.update(_own_buffers(rl, s))
    if c["op"] == "router":
        how = dict(sigmoid=c["score"] == "sigmoid", normalize=c["normalize"], scale=s["scale"], balance_coef=s["coef"], valid=s["valid"])
        if c["dir"] == "fwd":
            return rl.relibra_router_fwd(s["logits"], s["ids"], **how, **b)
        return (rl.relibra_router_bwd(s["logits"], s["ids"], s["dgates"], s["counts"], s["n_valid"], s["dloss"], **how, **b),)
    if c["op"] == "block_norm":
        how = dict(y=s["y"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"], res_scale=s["res_scale"], eps=s["eps"])
        if c["dir"] == "fwd":
            outs = rl.relibra_block_norm_fwd(s["x"], **how, **b)
        else:
            outs = rl.relibra_block_norm_bwd(s["x"], s["dx_out"], s["dn"], **how, **b)
        return tuple(o for o in outs if o is not None)
    outs = rl.relibra_orthogonalize(s["grad"], momentum=s["momentum"], mu=s["mu"], nesterov=c["nesterov"], scale=s["scale"], **b)
    return tuple(o for o in outs if o is not None)


def _own_buffers(rl, s):
    c = s["case"]
    if c["op"] == "router":
        n_mb, T, k, E = c["n_mb"], c["T"], c["k"], c["E"]
        f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEV)
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=DEV)
        if c["dir"] == "bwd":
            return dict(dlogits=torch.empty_like(s["logits"]), err_flag=rl.new_err_flag())
        return dict(gates=f32(n_mb, T, k), counts=i32(n_mb, E), n_valid=i32(n_mb), prob_mean=f32(n_mb, E), loss=f32(n_mb),
                    workspace=rl.router_workspace(n_mb, T, k, E), err_flag=rl.new_err_flag())
    if c["op"] == "block_norm":
        x, h = s["x"], c["h"]
        if c["dir"] == "fwd":
            return dict(x_out=torch.empty_like(x), n=torch.empty_like(s["y"]) if c["pre"] else None)
        grad = lambda w: None if w is None else torch.empty(h, dtype=torch.float32, device=DEV)
        return dict(dx=torch.empty_like(x), dy=torch.empty_like(s["y"]), dgate=None if s["gate"] is None else torch.empty_like(s["gate"]),
                    dw_post=grad(s["w_post"]), dw_pre=grad(s["w_pre"]), workspace=rl.block_norm_workspace(c["T"], h))
    return dict(out=torch.empty(s["grad"].shape, dtype=torch.bfloat16, device=DEV),
                momentum_out=None if s["momentum"] is None else torch.empty_like(s["momentum"]),
                workspace=rl.orthogonalize_workspace(c["blocks"], c["rows"], c["cols"]))


# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definition in double precision, from the inputs alone: one micro-batch, row or matrix at a time where that keeps memory
    small, with formulas other than the plain form's."""
    s = prepare(case, seed)
    if case["op"] == "router":
        return _router_exact(s)
    if case["op"] == "block_norm":
        return _norm_exact(s)
    return _ortho_exact(s)


def _router_exact(s):
    c = s["case"]
    E, k = c["E"], c["k"]
    outs = []
    for mb in range(c["n_mb"]):
        z, ids = s["logits"][mb].double(), s["ids"][mb].long()
        live = torch.ones(c["T"], dtype=torch.bool, device=DEV) if s["valid"] is None else s["valid"][mb] != 0
        # weights instead of log scores: exp(z), shifted per token, or the sigmoid itself
        w = torch.exp(z - z.amax(1, keepdim=True)) if c["score"] == "softmax" else torch.sigmoid(z)
        p = w / w.sum(1, keepdim=True)
        ws = torch.gather(w, 1, ids)
        total = ws.sum(1, keepdim=True) if c["normalize"] else (w.sum(1, keepdim=True) if c["score"] == "softmax" else torch.ones_like(ws[:, :1]))
        part = torch.where(total > 0, ws / total, torch.zeros_like(ws))
        n = int(live.sum())
        if c["dir"] == "fwd":
            counts = torch.bincount(ids[live].reshape(-1), minlength=E)
            mean = p[live].sum(0) / max(n, 1)
            loss = s["coef"] * E * (counts.double() * mean).sum() / (k * max(n, 1))
            outs.append((s["scale"] * part * live[:, None], counts.to(torch.int32), torch.tensor(n, dtype=torch.int32, device=DEV), mean, loss))
            continue
        # loss and gates as functions of the weights w: dL/dw, then dw/dz = w (softmax) or w (1 - sigmoid)
        cost = s["dloss"][mb].double() * s["coef"] * E * s["counts"][mb].double() / (k * max(n, 1)) / max(n, 1)
        dg = s["scale"] * s["dgates"][mb].double()
        grad = p * (cost[None, :] - (p @ cost)[:, None])                    # w * dL/dw
        sel = part * dg
        if c["normalize"]:
            sel = sel - part * sel.sum(1, keepdim=True)
        elif c["score"] == "softmax":
            grad = grad - p * sel.sum(1, keepdim=True)
        for j in range(k):
            grad[torch.arange(c["T"], device=DEV), ids[:, j]] += sel[:, j]
        if c["score"] == "sigmoid":
            grad = grad * torch.sigmoid(-z)
        outs.append((torch.where(live[:, None], grad, torch.zeros_like(grad)),))
    return tuple(torch.stack(o) for o in zip(*outs))


def _norm_exact(s):
    """x' and n from their definition; gradients from torch's own differentiation of it in double precision."""
    c = s["case"]
    rows = 1024
    acc = None
    parts = []
    for t0 in range(0, c["T"], rows):
        cut = slice(t0, t0 + rows)
        d = lambda name: None if s[name] is None else s[name].double()
        y = s["y"][cut].double().requires_grad_(True)
        w2, w1 = (None if w is None else w.requires_grad_(True) for w in (d("w_post"), d("w_pre")))
        gate = None if s["gate"] is None else s["gate"][cut].double().requires_grad_(True)
        norm = lambda v, w: v * torch.rsqrt(v.pow(2).sum(1, keepdim=True) / c["h"] + s["eps"]) * w
        z = y if w2 is None else norm(y, w2)
        z = z if gate is None else (gate[:, None] if gate.dim() == 1 else gate) * z
        if c["dir"] == "fwd":
            x_out = s["res_scale"] * s["x"][cut].double() + z
            parts.append(tuple(v.detach() for v in ((x_out,) if w1 is None else (x_out, norm(x_out, w1)))))
            continue
        # the saved stream's value with the block's dependence on x and y: x' = x_saved + res_scale * dx + (z - z0)
        dx = torch.zeros_like(y, requires_grad=True)
        x_out = s["x"][cut].double() + s["res_scale"] * dx + (z - z.detach())
        goal = (x_out * s["dx_out"][cut].double()).sum()
        if w1 is not None:
            goal = goal + (norm(x_out, w1) * s["dn"][cut].double()).sum()
        leaves = [v for v in (dx, y, gate, w2, w1) if v is not None]
        grads = list(torch.autograd.grad(goal, leaves))
        n_rows = 2 + (gate is not None)
        parts.append(tuple(grads[:n_rows]))
        acc = grads[n_rows:] if acc is None else [a + g for a, g in zip(acc, grads[n_rows:])]
    whole = tuple(torch.cat(o) for o in zip(*parts))
    return whole if acc is None else whole + tuple(acc)


def _ortho_exact(s):
    """The steps matrix by matrix, tall ones as they are (products from the right), A^2 X as A (A X)."""
    c = s["case"]
    outs, moms = [], []
    for b in range(c["blocks"]):
        g = s["grad"][b].double()
        u = g
        if s["momentum"] is not None:
            mom = s["mu"] * s["momentum"][b].double() + g
            moms.append(mom)
            u = g + s["mu"] * mom if c["nesterov"] else mom
        x = u / u.norm() if u.any() else u
        for _ in range(5):
            if c["rows"] <= c["cols"]:
                a = x @ x.T
                x = NS_A * x + NS_B * (a @ x) + NS_C * (a @ (a @ x))
            else:
                a = x.T @ x
                x = NS_A * x + NS_B * (x @ a) + NS_C * ((x @ a) @ a)
        outs.append(s["scale"] * x)
    return (torch.stack(outs),) + ((torch.stack(moms),) if moms else ())
