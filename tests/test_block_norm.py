"""The norms around a block with the residual stream between them, and their gradients, against plain double precision.

Tolerances.  A row's sum of h squares is taken in fp32 in at most h / 512 + 16 additions one behind the other; with the root and
the division a row's factor is off by less than (h / 512 + 24) 2^-24 of itself.  Everything else is a handful of products and sums,
held against the size of their terms; ROUNDINGS = h / 512 + 48 steps of 2^-24 cover a result.  One stored in bf16 is off by
another half step, 2^-8 of its value.  The stream is stored before its norm is taken from the unrounded values, so nothing of
its rounding reaches n.  A weight gradient's T terms are added in at most T / 16 + 64 additions one behind the other."""
import ctypes as C

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
U32 = torch.finfo(torch.float32).eps / 2
HALF16 = torch.finfo(torch.bfloat16).eps / 2


def make(T, h, stream=torch.bfloat16, post=True, pre=True, gate="token", has_y=True, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    b = lambda t: t.to(torch.bfloat16)
    d = dict(x=(size * r(T, h)).to(stream), y=b(size * r(T, h)) if has_y else None, w_post=b(1 + 0.3 * r(h)) if post and has_y else None,
             w_pre=b(1 + 0.3 * r(h)) if pre else None, dx_out=r(T, h).to(stream), dn=b(r(T, h)) if pre else None)
    d["gate"] = None if gate == "none" or not has_y else (torch.sigmoid(r(T)) if gate == "token" else b(torch.sigmoid(r(T, h))))
    return d


def rms(v, w, eps):
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * w


def forward(x, y, w_post, w_pre, gate, res_scale, eps):
    if y is None:
        return x, rms(x, w_pre, eps)
    z = y if w_post is None else rms(y, w_post, eps)
    if gate is not None:
        z = (gate[:, None] if gate.dim() == 1 else gate) * z
    x_out = res_scale * x + z
    return x_out, None if w_pre is None else rms(x_out, w_pre, eps)


def d64(t, grad=False):
    return None if t is None else t.double().requires_grad_(grad)


def dev(t):
    return None if t is None else t.to(DEV)


CASES = [
    dict(T=1, h=8), dict(T=3, h=512), dict(T=5, h=520), dict(T=70, h=1000, gate="element"), dict(T=1, h=4096, gate="none"), dict(T=9, h=8192, gate="element"),
    dict(T=33, h=2048, post=False), dict(T=33, h=2048, pre=False), dict(T=33, h=1024, post=False, pre=False), dict(T=17, h=768, has_y=False),
    dict(T=1100, h=1032), dict(T=1030, h=4104, gate="element"), dict(T=1025, h=8192, gate="none"), dict(T=5000, h=64, gate="element"), dict(T=2000, h=256, has_y=False),
    dict(T=1500, h=640, post=False, gate="none"), dict(T=21, h=88, gate="element", post=False),
    dict(T=300, h=8184, gate="element"), dict(T=4100, h=1536), dict(T=9000, h=200, gate="none"),
]
IDS = lambda c: "-".join(f"{k}{v}" for k, v in c.items())


@gpu
@pytest.mark.parametrize("kw", CASES, ids=IDS)
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_block_norm_against_the_definition(kw, stream):
    d = make(stream=stream, **kw)
    T, h, s, eps = kw["T"], kw["h"], 0.75, 1e-5
    half = torch.finfo(stream).eps / 2
    rel = (h / 512 + 48) * U32
    how = {k: dev(d[k]) for k in ("y", "w_post", "w_pre", "gate")}
    x_out, n = rl.relibra_block_norm_fwd(dev(d["x"]), **how, res_scale=s, eps=eps)
    with torch.no_grad():
        want = forward(*(d64(d[k]) for k in ("x", "y", "w_post", "w_pre", "gate")), s, eps)
        terms = forward(*(d64(d[k]).abs() if d[k] is not None else None for k in ("x", "y", "w_post", "w_pre", "gate")), s, eps)[0]
        if d["y"] is not None:
            off = (x_out.cpu().double() - want[0]).abs()
            assert torch.all(off <= half * want[0].abs() + rel * terms), float(off.max())
        if n is None:
            assert d["w_pre"] is None
        else:
            size = terms / torch.sqrt((want[0] ** 2).mean(1, keepdim=True) + eps) * d64(d["w_pre"]).abs()
            off = (n.cpu().double() - want[1]).abs()
            assert torch.all(off <= HALF16 * want[1].abs() + 2 * rel * (size + want[1].abs())), float(off.max())
    # backward, from the stored stream
    check_backward(d, x_out.cpu(), s, eps, rel, half)


def check_backward(d, x_out, s, eps, rel, half, **given):
    T, h = x_out.shape
    how = {k: dev(d[k]) for k in ("y", "w_post", "w_pre", "gate")}
    got = rl.relibra_block_norm_bwd(dev(x_out), dev(d["dx_out"]), dev(d["dn"]), **how, res_scale=s, eps=eps, **given)
    y, w2, w1, gate = (d64(d[k], True) for k in ("y", "w_post", "w_pre", "gate"))
    step = torch.zeros((T, h), dtype=torch.float64, requires_grad=True)       # d/dx at the stored stream
    z = None if y is None else (y if w2 is None else rms(y, w2, eps))
    if z is not None and gate is not None:
        z = (gate[:, None] if gate.dim() == 1 else gate) * z
    xo = d64(x_out) + (s if y is not None else 1.0) * step + (0 if z is None else z - z.detach())
    goal = (xo * (0 if d["dx_out"] is None else d64(d["dx_out"]))).sum()
    if w1 is not None:
        goal = goal + (rms(xo, w1, eps) * d64(d["dn"])).sum()
    goal.backward()
    with torch.no_grad():
        # sizes of the terms
        A = torch.zeros((T, h), dtype=torch.float64) if d["dx_out"] is None else d64(d["dx_out"]).abs()
        if w1 is not None:
            r1 = 1 / torch.sqrt((d64(x_out) ** 2).mean(1, keepdim=True) + eps)
            xh, wn = (d64(x_out) * r1).abs(), (w1 * d64(d["dn"])).abs()
            A = A + r1 * (wn + xh * (wn * xh).mean(1, keepdim=True))
        names = ["dx", "dy", "dgate", "dw_post", "dw_pre"]
        wants = [step.grad, None if y is None else y.grad, None if gate is None else gate.grad, None if w2 is None else w2.grad, None if w1 is None else w1.grad]
        sizes = [A, None, None, None, None]
        if y is not None:
            g = 1.0 if gate is None else (gate[:, None] if gate.dim() == 1 else gate).abs()
            r2 = 1 / torch.sqrt((y * y).mean(1, keepdim=True) + eps) if w2 is not None else 1.0
            yh = (y * r2).abs()
            ww = 1.0 if w2 is None else w2.abs()
            sizes[1] = g * A if w2 is None else r2 * (g * A * ww + yh * (g * A * ww * yh).mean(1, keepdim=True))
            if gate is not None:
                sizes[2] = (A * yh * ww).sum(1) if gate.dim() == 1 else A * yh * ww
            if w2 is not None:
                sizes[3] = (g * A * yh).sum(0)
        if w1 is not None:
            sizes[4] = (d64(d["dn"]).abs() * xh).sum(0)
        halves = [half, HALF16, U32 if gate is not None and gate.dim() == 1 else HALF16, U32, U32]
        for i, name in enumerate(names):
            if wants[i] is None:
                assert got[i] is None
                continue
            tol = halves[i] * wants[i].abs() + 2 * (rel + (T / 16 + 64) * U32 * (i >= 3)) * sizes[i] + 1e-30
            off = (got[i].cpu().double() - wants[i]).abs()
            assert torch.all(off <= tol), (name, float(off.max()), float((off / tol).max()))
    return got


@gpu
def test_block_norm_gradient_against_differences():
    """Central differences of the library's own forward pass in an fp32 stream."""
    T, h, eps, s = 3, 16, 1e-3, 0.5
    d = make(T, h, torch.float32, seed=4)
    n_up, x_up = d["dn"].double(), d["dx_out"].double()
    how = {k: dev(d[k]) for k in ("w_post", "w_pre", "gate")}
    x, y = dev(d["x"]), dev(d["y"])
    x_out, _ = rl.relibra_block_norm_fwd(x, y=y, **how, res_scale=s, eps=eps)
    dx = rl.relibra_block_norm_bwd(x_out, dev(d["dx_out"]), dev(d["dn"]), y=y, **how, res_scale=s, eps=eps)[0].cpu().double()
    step = 2.0 ** -4

    def value(xx):
        xo, n = rl.relibra_block_norm_fwd(xx, y=y, **how, res_scale=s, eps=eps)
        return float((xo.cpu().double() * x_up).sum()), n.cpu().double()
    for t in range(T):
        for c in range(h):
            up, dn = x.clone(), x.clone()
            up[t, c] += step
            dn[t, c] -= step
            (a, na), (b, nb) = value(up), value(dn)
            diff = ((a - b) + ((na - nb) * n_up).sum().item()) / (2 * step)
            # n in bf16: half a step of values of up to 4 on h values, twice; third derivative below 10 per unit of dn
            noise = 2 * 4 * HALF16 * n_up[t].abs().sum().item() / (2 * step)
            assert abs(diff - float(dx[t, c])) <= noise + 10 * step * step / 6 * n_up[t].abs().sum().item()


@gpu
def test_block_norm_accumulates_and_drops_absent_upstreams():
    d = make(300, 264, torch.bfloat16, gate="element", seed=8)
    how = {k: dev(d[k]) for k in ("y", "w_post", "w_pre", "gate")}
    x_out, _ = rl.relibra_block_norm_fwd(dev(d["x"]), **how)
    once = rl.relibra_block_norm_bwd(x_out, dev(d["dx_out"]), dev(d["dn"]), **how)
    w2, w1 = once[3].clone() + 5, once[4].clone() - 3
    twice = rl.relibra_block_norm_bwd(x_out, dev(d["dx_out"]), dev(d["dn"]), **how, accumulate=True, dw_post=w2, dw_pre=w1)
    assert torch.equal(twice[3], (once[3] + 5) + once[3]) and torch.equal(twice[4], (once[4] - 3) + once[4]) and twice[3] is w2
    rel = (264 / 512 + 48) * U32
    check_backward(dict(d, dx_out=None), x_out.cpu(), 1.0, 1e-6, rel, HALF16)
    # T = 0: gradients are zeros, or stay as they are
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)
    how0 = dict(y=e(0, 264), w_post=how["w_post"], w_pre=how["w_pre"])
    assert rl.relibra_block_norm_fwd(e(0, 264), **how0)[1].shape == (0, 264)
    got = rl.relibra_block_norm_bwd(e(0, 264), e(0, 264), e(0, 264), **how0)
    assert got[3].abs().sum() == 0 and got[4].abs().sum() == 0
    got = rl.relibra_block_norm_bwd(e(0, 264), e(0, 264), e(0, 264), **how0, accumulate=True, dw_post=w2, dw_pre=w1)
    assert torch.equal(got[3], twice[3])


@gpu
def test_block_norm_rows_of_zeros_large_values_and_nan():
    d = make(40, 512, torch.float32, gate="none", seed=12)
    d["y"][3], d["x"][3] = 0, 0                              # nothing in the row: n is 0
    d["y"][5] = 1e17                                         # squares reach 1e34
    d["x"][7] = float("nan")
    x_out, n = rl.relibra_block_norm_fwd(dev(d["x"]), **{k: dev(d[k]) for k in ("y", "w_post", "w_pre")})
    assert torch.all(n[3] == 0) and torch.isfinite(n[5].float()).all()
    assert torch.isnan(n[7].float()).all() and torch.isfinite(torch.cat([n[:7], n[8:]]).float()).all()
    got = rl.relibra_block_norm_bwd(x_out, dev(d["dx_out"]), dev(d["dn"]), **{k: dev(d[k]) for k in ("y", "w_post", "w_pre")})
    for g in got[:2]:
        assert torch.isnan(g[7].float()).any() and torch.isfinite(torch.cat([g[:7], g[8:]]).float()).all()


@gpu
def test_block_norm_in_place():
    d = make(600, 1024, torch.bfloat16, seed=14)
    how = {k: dev(d[k]) for k in ("w_post", "w_pre", "gate")}
    x, y = dev(d["x"]), dev(d["y"])
    want = rl.relibra_block_norm_fwd(x, y=y, **how)
    wb = rl.relibra_block_norm_bwd(want[0], dev(d["dx_out"]), dev(d["dn"]), y=y, **how)
    xi, yi = x.clone(), y.clone()
    got = rl.relibra_block_norm_fwd(xi, y=yi, **how, x_out=xi, n=yi)
    assert got[0] is xi and torch.equal(xi, want[0]) and torch.equal(yi, want[1])
    di, yi = dev(d["dx_out"]), y.clone()
    got = rl.relibra_block_norm_bwd(want[0], di, dev(d["dn"]), y=yi, **how, dx=di, dy=yi)
    assert all(torch.equal(a, b) for a, b in zip(got, wb))


@gpu
def test_block_norm_in_a_graph_beside_eager_calls():
    d = make(1300, 1024, torch.bfloat16, gate="element", seed=16)
    how = {k: dev(d[k]) for k in ("w_post", "w_pre", "gate", "y")}
    x, dxo, dn = dev(d["x"]), dev(d["dx_out"]), dev(d["dn"])
    ws = rl.block_norm_workspace(1300, 1024)

    def step(xx, **kw):
        x_out, n = rl.relibra_block_norm_fwd(xx, **how)
        return (x_out, n, *rl.relibra_block_norm_bwd(x_out, dxo, dn, **how, **kw))
    step(x, workspace=ws)
    src = x.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(src, workspace=ws)
    side = torch.cuda.Stream()
    for turn in range(3):
        src.copy_(x * (turn + 1))
        want = step(src.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step(src)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), turn


# ------------------------------------------------------------------ refusals (no GPU needed: nothing is launched)
P, F = C.c_void_p, C.c_float


def _fwd(x=4096, y=4096, w_post=4096, w_pre=4096, gate=4096, T=4, h=64, eps=1e-6, flags=2, x_out=4096, n=4096):
    return rl.lib().relibra_block_norm_fwd(P(x), P(y), P(w_post), P(w_pre), P(gate), T, h, F(1), F(eps), flags, P(x_out), P(n), P(0))


def _bwd(x=4096, dxo=4096, dn=4096, y=4096, w_post=4096, w_pre=4096, gate=4096, T=4, h=64, eps=1e-6, flags=2, dx=4096, dy=4096, dgate=4096, dw_post=4096, dw_pre=4096,
         ws=4096, ws_bytes=1 << 30):
    return rl.lib().relibra_block_norm_bwd(P(x), P(dxo), P(dn), P(y), P(w_post), P(w_pre), P(gate), T, h, F(1), F(eps), flags, P(dx), P(dy), P(dgate), P(dw_post),
                                           P(dw_pre), P(ws), C.c_size_t(ws_bytes), P(0))


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_block_norm_refusals(call):
    for bad in (dict(T=-1), dict(h=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(flags=16), dict(flags=6), dict(x=0), dict(gate=0), dict(x=4104), dict(y=4104),
                dict(w_post=4104), dict(w_pre=4104), dict(flags=4, gate=4100), dict(y=0), dict(y=0, w_post=0), dict(y=0, gate=0, flags=0), dict(y=0, w_post=0, w_pre=0, flags=0)):
        assert call(**bad) == rl.EINVAL, bad
    for bad in (dict(h=12), dict(h=8200), dict(T=(1 << 30) + 1)):
        assert call(**bad) == rl.EUNSUPPORTED, bad


def test_block_norm_refuses_missing_outputs_and_small_workspaces():
    assert _fwd(flags=8) == rl.EINVAL                        # nothing to accumulate in the forward pass
    assert _fwd(x_out=0) == rl.EINVAL and _fwd(n=0) == rl.EINVAL and _fwd(T=0) == rl.OK
    for bad in ("dn", "dx", "dy", "dgate", "dw_post", "dw_pre"):
        assert _bwd(**{bad: 0}) == rl.EINVAL, bad
    assert _bwd(w_pre=0, dxo=0) == rl.EINVAL and _bwd(flags=4, dgate=4100) == rl.EINVAL and _bwd(ws=4104) == rl.EINVAL
    need = rl.workspace_bytes(rl.WS_BLOCK_NORM, 4, 1, 1, 1, 64, 0)
    assert need > 0 and _bwd(ws_bytes=need - 1) == rl.EWORKSPACE and _bwd(ws=0) == rl.EWORKSPACE


@gpu
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_block_norm_rows_whose_squares_pass_fp32(stream):
    """sqrt(3.4e38 / 512) = 8e17: a row of 1e19 has an infinite rms and the norm 0, 1e17 is an ordinary row; no other row notices."""
    d = make(40, 512, stream, gate="none", seed=15)
    plain = rl.relibra_block_norm_fwd(dev(d["x"]), **{k: dev(d[k]) for k in ("y", "w_post", "w_pre")})
    d["y"][3], d["x"][5], d["x"][6] = 1e19, 1e19, 1e17
    x_out, n = rl.relibra_block_norm_fwd(dev(d["x"]), **{k: dev(d[k]) for k in ("y", "w_post", "w_pre")})
    assert torch.equal(x_out[3], dev(d["x"][3]))             # x + 0
    assert torch.all(n[5] == 0) and torch.all((n[6].float() / dev(d["w_pre"]).float() - 1).abs() <= 2 * HALF16)
    rest = [i for i in range(40) if i not in (3, 5, 6)]
    assert torch.equal(x_out[rest], plain[0][rest]) and torch.equal(n[rest], plain[1][rest])


# ------------------------------------------------------------------ outputs of NaN before the call, NaN around them
def guarded(shape, dtype):
    """A tensor of NaN with 64 elements of it in front and behind, and a check that those are as they were."""
    count = 1
    for s in shape:
        count *= s
    flat = torch.full((count + 128,), -1, dtype=torch.int16 if dtype.itemsize == 2 else torch.int32, device=DEV)
    return flat.view(dtype)[64:64 + count].view(shape), lambda: bool((torch.cat([flat[:64], flat[64 + count:]]) == -1).all())


@gpu
@pytest.mark.parametrize("kw", [dict(T=1, h=8), dict(T=601, h=200), dict(T=33, h=1032, gate="element"), dict(T=1027, h=4104), dict(T=7, h=8192, gate="none")], ids=IDS)
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_block_norm_writes_every_value_and_nothing_else(kw, stream):
    d = make(stream=stream, seed=18, **kw)
    T, h, b16, f32 = kw["T"], kw["h"], torch.bfloat16, torch.float32
    how = {k: dev(d[k]) for k in ("y", "w_post", "w_pre", "gate")}
    want = rl.relibra_block_norm_fwd(dev(d["x"]), **how)
    grads = rl.relibra_block_norm_bwd(want[0], dev(d["dx_out"]), dev(d["dn"]), **how)
    out = [guarded((T, h), stream), guarded((T, h), b16)]
    rl.relibra_block_norm_fwd(dev(d["x"]), **how, x_out=out[0][0], n=out[1][0])
    ws = torch.full((rl.workspace_bytes(rl.WS_BLOCK_NORM, T, 1, 1, 1, h, 0) + 256,), 255, dtype=torch.uint8, device=DEV)
    back = [guarded((T, h), stream), guarded((T, h), b16), None if d["gate"] is None else guarded(d["gate"].shape, d["gate"].dtype), guarded((h,), f32), guarded((h,), f32)]
    names = ("dx", "dy", "dgate", "dw_post", "dw_pre")
    rl.relibra_block_norm_bwd(want[0], dev(d["dx_out"]), dev(d["dn"]), **how, workspace=ws[:-256], **{k: v[0] for k, v in zip(names, back) if v})
    for (got, kept), w in zip(out + [v for v in back if v], list(want) + [v for v in grads if v is not None]):
        assert torch.equal(got, w) and kept() and torch.isfinite(got.float()).all()
    assert torch.all(ws[-256:] == 255)


@gpu
@pytest.mark.parametrize("kw", [dict(T=601, h=200), dict(T=5, h=4096), dict(T=1027, h=1536, gate="element")], ids=IDS)
def test_block_norm_gradient_over_its_upstream(kw):
    """dx in the place of dx_out, dy in that of dn; the last rows of a block are not all there."""
    d = make(stream=torch.float32, seed=19, **kw)
    how = {k: dev(d[k]) for k in ("y", "w_post", "w_pre", "gate")}
    x_out, _ = rl.relibra_block_norm_fwd(dev(d["x"]), **how)
    want = rl.relibra_block_norm_bwd(x_out, dev(d["dx_out"]), dev(d["dn"]), **how)
    dxo, dn = dev(d["dx_out"]), dev(d["dn"])
    got = rl.relibra_block_norm_bwd(x_out, dxo, dn, **how, dx=dxo, dy=dn)
    assert got[0] is dxo and got[1] is dn
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, want))
