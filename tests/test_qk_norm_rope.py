"""Norms of queries and keys for each head with the rotation by their positions, and the gradients, against plain double precision.

Tolerances.  A head's sum of d <= 256 squares is taken in fp32 in at most 20 additions one behind the other (16 values a lane, then 4
exchanges); with the root, the division, the weight and the turn's two products and sum ROUNDINGS = 40 steps of 2^-24 cover a value, held
against the size of its terms.  A cosine or sine in fp32 of a reduced angle in double is off by less than 4 steps and 2^-24 of a turn (2 pi):
another 12 steps.  What is stored in bf16 is off by half a step more, 2^-8 of its value.  A weight gradient's terms are added in at most T H + 16 additions
one behind the other, fewer by far in the kernel; (T / 8 + 64) steps cover what it does."""
import ctypes as C

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
BF16 = torch.bfloat16
U32 = torch.finfo(torch.float32).eps / 2
HALF16 = torch.finfo(BF16).eps / 2
REL = 52 * U32


def make(T, Hq, Hk, d, rot=None, axes=1, adjacent=False, norm=True, seed=0, far=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    b = lambda t: t.to(BF16)
    rot = d if rot is None else rot
    c = dict(q=b(r(T, Hq, d) * torch.exp(r(1, Hq, 1))), k=b(r(T, Hk, d)), up_q=b(r(T, Hq, d)), up_k=b(r(T, Hk, d)), adjacent=adjacent, eps=1e-5,
             w_q=b(1 + 0.3 * r(d)) if norm else None, w_k=b(1 + 0.3 * r(d)) if norm else None, pos=None, freq=None, axis=None)
    if rot:
        c["freq"] = (1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float()
        c["pos"] = torch.randint(-50, 5000, (axes, T), generator=g, dtype=torch.int32) + far
        c["axis"] = [int(a) for a in torch.randint(0, axes, (rot // 2,), generator=g)] if axes > 1 else None
    return c


def turn(x, c, sign=1):
    """Pairs turned by sign * angle, in double; x [T, H, d]."""
    if c["freq"] is None:
        return x
    half = c["freq"].numel()
    axis = torch.zeros(half, dtype=torch.long) if c["axis"] is None else torch.tensor(c["axis"])
    angle = (c["pos"].double()[axis].T * c["freq"].double())[:, None, :]
    a = torch.arange(half) * (2 if c["adjacent"] else 1)
    b = a + (1 if c["adjacent"] else half)
    y = x.clone()
    y[..., a] = x[..., a] * angle.cos() - sign * x[..., b] * angle.sin()
    y[..., b] = x[..., b] * angle.cos() + sign * x[..., a] * angle.sin()
    return y


def forward(x, w, c):
    x = x.double()
    return turn(x if w is None else x / torch.sqrt((x * x).mean(2, keepdim=True) + c["eps"]) * w.double(), c)


def sizes(x, c):
    """The size of a turn's terms: its pairs' magnitudes."""
    if c["freq"] is None:
        return x.abs()
    half = c["freq"].numel()
    a = torch.arange(half) * (2 if c["adjacent"] else 1)
    b = a + (1 if c["adjacent"] else half)
    y = x.abs().clone()
    y[..., a] = y[..., b] = (x[..., a] ** 2 + x[..., b] ** 2).sqrt() * 1.5
    return y


def dev(t):
    return None if t is None else t.to(DEV)


def how(c):
    return dict(pos=dev(c["pos"]), freq=dev(c["freq"]), w_q=dev(c["w_q"]), w_k=dev(c["w_k"]), axis=c["axis"], adjacent=c["adjacent"], eps=c["eps"])


CASES = [dict(T=1, Hq=1, Hk=1, d=16), dict(T=1, Hq=32, Hk=4, d=128), dict(T=5, Hq=3, Hk=1, d=32, rot=16), dict(T=77, Hq=12, Hk=12, d=80, rot=32, adjacent=True),
         dict(T=130, Hq=20, Hk=5, d=96, axes=3), dict(T=64, Hq=9, Hk=2, d=112, rot=48, axes=4, adjacent=True), dict(T=33, Hq=5, Hk=3, d=192, rot=96, axes=2),
         dict(T=19, Hq=17, Hk=9, d=256), dict(T=40, Hq=4, Hk=2, d=64, norm=False), dict(T=40, Hq=4, Hk=2, d=64, rot=0), dict(T=4100, Hq=2, Hk=1, d=48),
         dict(T=9000, Hq=1, Hk=1, d=16, adjacent=True), dict(T=30, Hq=4, Hk=2, d=128, far=1 << 30)]
IDS = lambda c: "-".join(f"{k}{v}" for k, v in c.items())


@gpu
@pytest.mark.parametrize("kw", CASES, ids=IDS)
def test_qk_norm_rope_against_the_definition(kw):
    c = make(**kw)
    got = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    for y, x, w in zip(got, (c["q"], c["k"]), (c["w_q"], c["w_k"])):
        want = forward(x, w, c)
        u = forward(x, w, dict(c, freq=None))
        off = (y.cpu().double() - want).abs()
        assert torch.all(off <= HALF16 * want.abs() + 2 * REL * sizes(u, c)), float(off.max())
    check_backward(c)


def check_backward(c, dw=None, **given):
    got = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c), **given)
    T = c["q"].shape[0]
    for i, (x, w, up) in enumerate(((c["q"], c["w_q"], c["up_q"]), (c["k"], c["w_k"], c["up_k"]))):
        leaf = x.double().requires_grad_(True)
        wl = None if w is None else w.double().requires_grad_(True)
        (forward(leaf, wl, c) * up.double()).sum().backward()
        g = sizes(turn(up.double(), c, -1), c)
        with torch.no_grad():
            if w is None:
                size = g
                assert got[2 + i] is None
            else:
                r = 1 / torch.sqrt((x.double() ** 2).mean(2, keepdim=True) + c["eps"])
                xh, wg = (x.double() * r).abs(), w.double().abs() * g
                size = r * (wg + xh * (wg * xh).mean(2, keepdim=True))
                off = (got[2 + i].cpu().double() - wl.grad).abs()
                assert torch.all(off <= U32 * wl.grad.abs() + (2 * REL + (T / 8 + 64) * U32) * (g * xh).sum((0, 1))), float(off.max())
            off = (got[i].cpu().double() - leaf.grad).abs()
            assert torch.all(off <= HALF16 * leaf.grad.abs() + 3 * REL * size), float(off.max())
    return got


@gpu
def test_qk_norm_rope_gradient_against_differences():
    """Central differences of the call itself: T = 2 tokens, outputs in bf16 (half a step of values of up to 4 on d values), steps of 1/8."""
    c = make(2, 2, 1, 16, seed=5)
    step = 0.125
    c["q"] = (c["q"].float() * 8).round().div(8).clamp(-4, 4).to(BF16)       # so that a step either way has no rounding
    dq = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))[0].cpu().double()
    value = lambda q: (rl.relibra_qk_norm_rope_fwd(dev(q), dev(c["k"]), **how(c))[0].cpu().double() * c["up_q"].double()).sum().item()
    for t, h, j in ((0, 0, 0), (0, 1, 9), (1, 0, 15), (1, 1, 3)):
        up, dn = c["q"].clone(), c["q"].clone()
        up[t, h, j] += step
        dn[t, h, j] -= step
        exact = lambda q: (forward(q, c["w_q"], c) * c["up_q"].double()).sum().item()
        noise = 2 * 6 * HALF16 * c["up_q"][t, h].double().abs().sum().item() / (2 * step)
        bend = abs((exact(up) - exact(dn)) / (2 * step) - dq[t, h, j].item())      # what the step's size itself leaves
        assert bend <= 0.5 + 0.02 * abs(dq[t, h, j].item())
        assert abs((value(up) - value(dn)) / (2 * step) - dq[t, h, j].item()) <= noise + bend


STEP = 0.125


def value(y_q, y_k, c):
    return (y_q.cpu().double() * c["up_q"].double()).sum().item() + (y_k.cpu().double() * c["up_k"].double()).sum().item()


def defined(c):
    return forward(c["q"], c["w_q"], c), forward(c["k"], c["w_k"], c)


def gradient_error(c, name, grad):
    """What the gradient of input `name` may be off by, as in check_backward."""
    x, w, up = (c[n] for n in (("q", "w_q", "up_q") if name in ("q", "w_q") else ("k", "w_k", "up_k")))
    g = sizes(turn(up.double(), c, -1), c)
    if w is None:
        return HALF16 * grad.abs() + 3 * REL * g
    r = 1 / torch.sqrt((x.double() ** 2).mean(2, keepdim=True) + c["eps"])
    xh, wg = (x.double() * r).abs(), w.double().abs() * g
    if name in ("w_q", "w_k"):
        return U32 * grad.abs() + (2 * REL + (x.shape[0] / 8 + 64) * U32) * (g * xh).sum((0, 1))
    return HALF16 * grad.abs() + 3 * REL * r * (wg + xh * (wg * xh).mean(2, keepdim=True))


def difference_case(kw, name):
    """Upstream for one side; for a weight of the normed head's own signs, so that what tokens and heads add to its gradient has one sign."""
    c = make(seed=15, **kw)
    c["up_k" if name in ("q", "w_q") else "up_q"].zero_()
    if name in ("w_q", "w_k"):
        up = "up_" + name[2]
        c[up] = turn(c[up].double().abs() * c[name[2]].double().sign(), c).to(BF16)
    return c


def differences(c, name, outputs):
    """(half the difference of the outputs' sum against the upstream one step along the signs of the definition's gradient of input `name` and one step back, how far it may be from the gradient's slope,
    the step, the gradient, how far the library's may be off).  Along the signs the slope is the sum of the gradient's sizes; what the curve adds to a central difference is the definition's own,
    what outputs and gradients are off by is the tolerance of the test against the definition."""
    leaves = {n: c[n].double().requires_grad_(True) for n in ("q", "k", "w_q", "w_k") if c[n] is not None}
    y = (forward(leaves["q"], leaves.get("w_q"), c), forward(leaves["k"], leaves.get("w_k"), c))
    ((y[0] * c["up_q"].double()).sum() + (y[1] * c["up_k"].double()).sum()).backward()
    grad = leaves[name].grad
    ends = [dict(c, **{name: (c[name].double() + s * STEP * grad.sign()).to(BF16)}) for s in (1, -1)]
    moved = (ends[0][name].double() - ends[1][name].double()) / 2
    slope = (moved * grad).sum().item()
    noise = 0.0
    for e in ends:
        for y, x, w, up in zip(defined(e), (e["q"], e["k"]), (e["w_q"], e["w_k"]), (e["up_q"], e["up_k"])):
            noise += ((HALF16 * y.abs() + 2 * REL * sizes(forward(x, w, dict(e, freq=None)), e)) * up.double().abs()).sum().item() / 2
    bend = abs((value(*defined(ends[0]), c) - value(*defined(ends[1]), c)) / 2 - slope)
    own = (moved.abs() * gradient_error(c, name, grad)).sum().item()
    return (value(*outputs(ends[0]), c) - value(*outputs(ends[1]), c)) / 2, 1.01 * (bend + noise + own), moved, grad


DIFFERENCES = [dict(T=2, Hq=2, Hk=1, d=16), dict(T=30, Hq=5, Hk=2, d=96, rot=32, axes=3), dict(T=9, Hq=4, Hk=3, d=128, adjacent=True), dict(T=20, Hq=3, Hk=2, d=64, norm=False)]
INPUTS = [(kw, name) for kw in DIFFERENCES for name in ("q", "k", "w_q", "w_k") if kw.get("norm", True) or name in ("q", "k")]


@gpu
@pytest.mark.parametrize("kw,name", INPUTS, ids=lambda x: IDS(x) if isinstance(x, dict) else x)
def test_qk_norm_rope_gradient_against_its_own_differences(kw, name):
    c = difference_case(kw, name)
    got = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))[("q", "k", "w_q", "w_k").index(name)].cpu().double()
    diff, tol, moved, _ = differences(c, name, lambda e: rl.relibra_qk_norm_rope_fwd(dev(e["q"]), dev(e["k"]), **how(e)))
    assert abs(diff - (moved * got).sum().item()) <= tol


@pytest.mark.parametrize("kw,name", INPUTS, ids=lambda x: IDS(x) if isinstance(x, dict) else x)
def test_qk_norm_rope_differences_tell_wrong_gradients(kw, name):
    """What the test above would say of other gradients, with the definition in the library's place: the right one passes; none, half of it, and one of the wrong sign do not, not even if
    everything that may be off were off in their favour."""
    c = difference_case(kw, name)
    diff, tol, moved, grad = differences(c, name, defined)
    right = (moved * grad).sum().item()
    assert abs(diff - right) <= tol
    for wrong in (0.0, 0.5, -1.0):
        assert abs(diff - wrong * right) > 2 * tol, (wrong, diff, right, tol)

@gpu
@pytest.mark.parametrize("kw", [dict(T=33, Hq=8, Hk=2, d=128), dict(T=700, Hq=3, Hk=2, d=80, rot=32, adjacent=True)], ids=IDS)
def test_qk_norm_rope_of_a_fused_projection(kw):
    """Parts of one tensor in, parts of one tensor out, in place and over the upstream: the same bits, and nothing beside them is written."""
    c = make(seed=2, **kw)
    T, Hq, Hk, d = kw["T"], kw["Hq"], kw["Hk"], kw["d"]
    want = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    back = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))

    def fused(q, k):
        whole = torch.full((T, (Hq + 2 * Hk) * d + 8), 7.0, dtype=BF16, device=DEV)
        parts = [p.unflatten(1, (-1, d)) for p in (whole[:, :Hq * d], whole[:, Hq * d:(Hq + Hk) * d])]
        parts[0].copy_(q)
        parts[1].copy_(k)
        return whole, parts
    whole, (q, k) = fused(c["q"], c["k"])
    got = rl.relibra_qk_norm_rope_fwd(q, k, **how(c))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dwhole, (gq, gk) = fused(c["up_q"], c["up_k"])
    dq, dk, dw_q, dw_k = rl.relibra_qk_norm_rope_bwd(q, k, gq, gk, **how(c), dq=gq, dk=gk)
    assert dq is gq and all(torch.equal(a, b) for a, b in zip((dq, dk, dw_q, dw_k), back))
    assert torch.all(dwhole[:, (Hq + Hk) * d:] == 7)
    got = rl.relibra_qk_norm_rope_fwd(q, k, **how(c), q_out=q, k_out=k)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.all(whole[:, (Hq + Hk) * d:] == 7)


@gpu
def test_qk_norm_rope_accumulates_and_takes_absent_parts():
    c = make(300, 6, 2, 64, seed=3)
    once = check_backward(c)
    w_q, w_k = once[2] + 5, once[3] - 3
    twice = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c), accumulate=True, dw_q=w_q, dw_k=w_k)
    assert torch.equal(twice[2], (once[2] + 5) + once[2]) and torch.equal(twice[3], (once[3] - 3) + once[3]) and twice[2] is w_q
    # one token: one block adds by itself
    c = make(1, 2, 1, 64, seed=4)
    once = check_backward(c)
    w_q, w_k = once[2] + 5, once[3] - 3
    rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c), accumulate=True, dw_q=w_q, dw_k=w_k)
    assert torch.equal(w_q, (once[2] + 5) + once[2]) and torch.equal(w_k, (once[3] - 3) + once[3])
    # queries alone; a norm on one side only
    c = make(50, 3, 2, 80, seed=6)
    full = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    h = {k: v for k, v in how(c).items() if k != "w_k"}
    alone = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), None, **h)
    assert alone[1] is None and torch.equal(alone[0], full[0])
    got = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), None, dev(c["up_q"]), None, **h)
    assert got[1] is None and got[3] is None
    half = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **h)
    assert torch.equal(half[0], full[0]) and torch.all((half[1].cpu().double() - forward(c["k"], None, c)).abs() <= HALF16 * forward(c["k"], None, c).abs() + 2 * REL * sizes(c["k"].double(), c))
    # no tokens: gradients of weights are zeros, or stay
    e = lambda H: torch.empty((0, H, 80), dtype=BF16, device=DEV)
    h = dict(how(c), pos=torch.empty((1, 0), dtype=torch.int32, device=DEV))
    assert rl.relibra_qk_norm_rope_fwd(e(3), e(2), **h)[0].shape == (0, 3, 80)
    got = rl.relibra_qk_norm_rope_bwd(e(3), e(2), e(3), e(2), **h)
    assert got[2].abs().sum() == 0 and got[3].abs().sum() == 0
    kept = got[2] + 2
    rl.relibra_qk_norm_rope_bwd(e(3), e(2), e(3), e(2), **h, accumulate=True, dw_q=kept, dw_k=got[3])
    assert torch.all(kept == 2)


@gpu
def test_qk_norm_rope_zeros_and_nan_stay_in_their_head():
    c = make(20, 4, 2, 64, seed=7)
    plain = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    c["q"][3, 1], c["q"][5, 2, 7] = 0, float("nan")
    got = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    assert torch.all(got[0][3, 1] == 0) and torch.isnan(got[0][5, 2].float()).all() and torch.equal(got[1], plain[1])
    rest = torch.ones(20, 4, dtype=torch.bool)
    rest[3, 1] = rest[5, 2] = False
    assert torch.equal(got[0][rest.to(DEV)], plain[0][rest.to(DEV)])
    back = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))
    assert torch.isfinite(back[0][3, 1].float()).all() and torch.isnan(back[0][5, 2].float()).all() and torch.isfinite(back[0][rest.to(DEV)].float()).all()


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
def test_qk_norm_rope_heads_whose_squares_pass_fp32(d):
    """sqrt(3.4e38 / 256) = 1.1e18: a head of 1e19 or 3e38 has an infinite rms, its norm and its gradients are zeros; one of 1e17 is an ordinary head; no other head notices."""
    c = make(12, 4, 2, d, seed=13)
    g = torch.Generator().manual_seed(14)
    sign = lambda: torch.randn(d, generator=g).sign()
    heads = (("q", 3, 1, 1e19), ("q", 5, 0, 3e38), ("k", 7, 1, 3e38), ("q", 9, 2, 1e17))
    for name, t, h, size in heads:
        c[name][t, h] = (size * sign()).to(BF16)
        c["up_" + name][t, h] = (4 * c["up_" + name][t, h].abs().float() * c[name][t, h].float().sign()).to(BF16)      # products of one sign: their sum passes fp32 for 3e38
    c["freq"].zero_()                                         # no turn: the upstream's signs are the norm's
    got = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    dx = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))
    for name, i in (("q", 0), ("k", 1)):
        x, w, up, y = c[name], c["w_" + name], c["up_" + name], got[i].cpu().double()
        leaf, wl = x.double().requires_grad_(True), w.double().requires_grad_(True)
        kept = torch.ones(x.shape[:2], dtype=torch.bool)
        for n, t, h, size in heads:
            if n == name and size > 1e18:
                kept[t, h] = False
                assert torch.all(y[t, h] == 0) and torch.all(dx[i][t, h] == 0), (n, size)
        want = forward(leaf, wl, c)
        (want * up.double())[kept].sum().backward()
        want = want.detach()
        assert torch.all((y - want).abs()[kept] <= (HALF16 + 2 * REL) * want.abs()[kept])
        with torch.no_grad():
            r = 1 / torch.sqrt((x.double() ** 2).mean(2, keepdim=True) + c["eps"])
            xh, wg = (x.double() * r).abs(), w.double().abs() * up.double().abs()
            size = r * (wg + xh * (wg * xh).mean(2, keepdim=True))
        assert torch.all((dx[i].cpu().double() - leaf.grad).abs()[kept] <= (HALF16 * leaf.grad.abs() + 3 * REL * size)[kept])
        off = (dx[2 + i].cpu().double() - wl.grad).abs()
        assert torch.all(off <= U32 * wl.grad.abs() + (2 * REL + 66 * U32) * (up.double().abs() * xh)[kept].sum(0)), float(off.max())

@gpu
def test_qk_norm_rope_writes_every_value_and_nothing_else():
    for kw in (dict(T=3, Hq=5, Hk=1, d=48), dict(T=1030, Hq=2, Hk=2, d=96, rot=32)):
        c = make(seed=8, **kw)
        T, d = kw["T"], kw["d"]
        want = (*rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c)), *rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c)))
        outs = []
        for w in (*want,):
            flat = torch.full((w.numel() + 128,), float("nan"), dtype=w.dtype, device=DEV)
            outs.append((flat, flat[64:-64].view(w.shape)))
        ws = torch.full((rl.workspace_bytes(rl.WS_QK_NORM_ROPE, T, 1, kw["Hq"], 1, kw["Hk"], d) + 256,), 255, dtype=torch.uint8, device=DEV)
        rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c), q_out=outs[0][1], k_out=outs[1][1])
        rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c), dq=outs[2][1], dk=outs[3][1], dw_q=outs[4][1], dw_k=outs[5][1], workspace=ws[:-256])
        for (flat, got), w in zip(outs, want):
            assert torch.equal(got, w) and torch.isnan(flat[:64].float()).all() and torch.isnan(flat[-64:].float()).all()
        assert torch.all(ws[-256:] == 255)


@gpu
def test_qk_norm_rope_in_a_graph_beside_eager_calls():
    c = make(1300, 8, 2, 128, seed=9)
    h = how(c)
    q, k, uq, uk = (dev(c[n]) for n in ("q", "k", "up_q", "up_k"))
    ws = rl.qk_norm_rope_workspace(1300, 8, 2, 128)

    def step(q, **kw):
        return (*rl.relibra_qk_norm_rope_fwd(q, k, **h), *rl.relibra_qk_norm_rope_bwd(q, k, uq, uk, **h, **kw))
    step(q, workspace=ws)
    src = q.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(src, workspace=ws)
    side = torch.cuda.Stream()
    for i in range(3):
        src.copy_(q * (i + 1))
        want = step(src.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step(src)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), i


@gpu
def test_qk_norm_rope_past_32_bits_of_offset():
    """Tokens 2^20 values apart: the last ones lie beyond 2^31 values from the first."""
    T, stride = 2300, 1 << 20
    c = make(T, 3, 2, 64, seed=11)
    want = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c))
    back = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c))
    whole = torch.empty((T, stride), dtype=BF16, device=DEV)
    q, k, uq, uk, oq, ok = (whole[:, a:a + h * 64].unflatten(1, (h, 64)) for a, h in ((0, 3), (192, 2), (1 << 19, 3), ((1 << 19) + 192, 2), (1024, 3), (1216, 2)))
    for to, name in ((q, "q"), (k, "k"), (uq, "up_q"), (uk, "up_k")):
        to.copy_(dev(c[name]))
    got = rl.relibra_qk_norm_rope_fwd(q, k, **how(c), q_out=oq, k_out=ok)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = rl.relibra_qk_norm_rope_bwd(q, k, uq, uk, **how(c), dq=oq, dk=uk)
    assert all(torch.equal(a, b) for a, b in zip(got, back))


# ------------------------------------------------------------------ refusals (no GPU needed: nothing is launched)
P, F, L = C.c_void_p, C.c_float, C.c_int64
M = 1 << 24                                                  # pretended tensors lie far apart


def _fwd(q=M, ql=256, k=2 * M, kl=128, w_q=4096, w_k=4096, pos=4096, freq=4096, axis=None, n_axes=1, T=4, Hq=4, Hk=2, d=64, rot=64, eps=1e-6, flags=0, qo=3 * M, qol=256, ko=4 * M, kol=128):
    return rl.lib().relibra_qk_norm_rope_fwd(P(q), L(ql), P(k), L(kl), P(w_q), P(w_k), P(pos), P(freq), axis, n_axes, T, Hq, Hk, d, rot, F(eps), flags, P(qo), L(qol), P(ko), L(kol), P(0))


def _bwd(q=M, ql=256, k=2 * M, kl=128, gq=5 * M, gql=256, gk=6 * M, gkl=128, w_q=4096, w_k=4096, pos=4096, freq=4096, axis=None, n_axes=1, T=4, Hq=4, Hk=2, d=64, rot=64, eps=1e-6, flags=0,
         qo=3 * M, qol=256, ko=4 * M, kol=128, dw_q=4096, dw_k=4096, ws=4096, ws_bytes=1 << 30):
    return rl.lib().relibra_qk_norm_rope_bwd(P(q), L(ql), P(k), L(kl), P(gq), L(gql), P(gk), L(gkl), P(w_q), P(w_k), P(pos), P(freq), axis, n_axes, T, Hq, Hk, d, rot, F(eps), flags,
                                             P(qo), L(qol), P(ko), L(kol), P(dw_q), P(dw_k), P(ws), C.c_size_t(ws_bytes), P(0))


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_qk_norm_rope_refusals(call):
    for bad in (dict(T=-1), dict(Hq=0), dict(Hk=-1), dict(d=0), dict(rot=-16), dict(rot=80), dict(flags=4), dict(eps=0.0), dict(eps=float("nan")), dict(w_q=4104), dict(w_k=4100),
                dict(rot=0, w_q=0, w_k=0), dict(pos=0), dict(freq=0), dict(n_axes=0), dict(Hk=0), dict(q=0), dict(k=0), dict(qo=0), dict(ko=0), dict(q=M + 8), dict(ql=255), dict(ql=260),
                dict(kl=120), dict(qol=248), dict(kol=(1 << 28) + 8), dict(qo=M, qol=512), dict(qo=M + 512), dict(ko=M), dict(qo=2 * M, qol=256), dict(qo=4 * M)):
        assert call(**bad) == rl.EINVAL, bad
    for bad in (dict(d=72), dict(d=272), dict(rot=24), dict(n_axes=5), dict(T=(1 << 30) + 1), dict(Hq=4097), dict(Hk=4097)):
        assert call(**bad) == rl.EUNSUPPORTED, bad
    assert call(axis=bytes([0] * 31 + [2]), n_axes=2) == rl.ERANGE
    assert call(T=0, q=0, k=0, qo=0, ko=0) == rl.OK if call is _fwd else True


def test_qk_norm_rope_backward_refuses_missing_outputs_and_small_workspaces():
    for bad in (dict(gq=0), dict(gk=0), dict(dw_q=0), dict(dw_k=0), dict(dw_q=4104), dict(ws=4104), dict(gql=255), dict(qo=6 * M), dict(ko=5 * M), dict(ko=M), dict(qo=5 * M + 16)):
        assert _bwd(**bad) == rl.EINVAL, bad
    assert _fwd(flags=2) == rl.EINVAL                        # nothing to accumulate in the forward pass
    need = rl.workspace_bytes(rl.WS_QK_NORM_ROPE, 4, 1, 4, 1, 2, 64)
    assert need > 0 and _bwd(ws_bytes=need - 1) == rl.EWORKSPACE and _bwd(ws=0) == rl.EWORKSPACE
    assert rl.workspace_bytes(rl.WS_QK_NORM_ROPE, 4, 1, 4, 1, 2, 72) == 0


def test_qk_norm_rope_refuses_overlaps_of_weights_tables_and_sums():
    """Every output against everything else that the call reads or writes, all of it apart but for the one pair."""
    at = {n: (100 + i) << 16 for i, n in enumerate(("w_q", "w_k", "pos", "freq"))}
    for name, a in at.items():                               # T = 4: rows of 512 and 256 bytes; weights and 32 frequencies 128 bytes, positions 16
        for out in ("qo", "ko"):
            assert _fwd(**dict(at, **{out: a})) == rl.EINVAL, (name, out)
    assert _fwd(**dict(at, w_q=3 * M - 112)) == rl.EINVAL and _fwd(**dict(at, pos=3 * M + 2044)) == rl.EINVAL and _fwd(**dict(at, freq=4 * M + 1020)) == rl.EINVAL
    need = rl.workspace_bytes(rl.WS_QK_NORM_ROPE, 4, 1, 4, 1, 2, 64)
    sums = {n: (200 + i) << 16 for i, n in enumerate(("dw_q", "dw_k", "ws"))}
    rows = dict(q=M, k=2 * M, gq=5 * M, gk=6 * M, qo=3 * M, ko=4 * M)
    apart = dict(at, **sums, ws_bytes=need)
    for flags in (0, rl.QK_ACCUMULATE):
        for name, a in sums.items():
            for other, b in {**at, **rows, **sums}.items():
                if other != name:
                    assert _bwd(**dict(apart, flags=flags, **{name: b})) == rl.EINVAL, (name, other)
        assert _bwd(**dict(apart, flags=flags, dw_q=sums["dw_k"] + 240)) == rl.EINVAL and _bwd(**dict(apart, flags=flags, dw_k=sums["ws"] + need - 16)) == rl.EINVAL
        assert _bwd(**dict(apart, flags=flags, T=0, dw_q=sums["dw_k"])) == rl.EINVAL
    for name, a in at.items():
        for out in ("qo", "ko"):
            assert _bwd(**dict(apart, **{out: a})) == rl.EINVAL, (name, out)


@gpu
def test_qk_norm_rope_takes_memory_between_its_rows():
    """Weights, tables and their gradients in the gaps between the rows of the outputs: shared by no row, and left or written as they should be."""
    c = make(9, 3, 2, 64, seed=12)
    want = (*rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **how(c)), *rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **how(c)))
    whole = torch.zeros((9, 1024), dtype=BF16, device=DEV)
    q, k = whole[:, :192].unflatten(1, (3, 64)), whole[:, 192:320].unflatten(1, (2, 64))
    h = how(c)
    gaps = dict(w_q=whole[0, 320:384], w_k=whole[1, 320:384], pos=whole[2, 320:338].view(torch.int32)[None], freq=whole[3, 320:384].view(torch.float32))
    for name, gap in gaps.items():
        gap.copy_(h[name])
        h[name] = gap
    got = rl.relibra_qk_norm_rope_fwd(dev(c["q"]), dev(c["k"]), **h, q_out=q, k_out=k)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    sums = [whole[r, 320:448].view(torch.float32) for r in (5, 6)]
    got = rl.relibra_qk_norm_rope_bwd(dev(c["q"]), dev(c["k"]), dev(c["up_q"]), dev(c["up_k"]), **h, dq=q, dk=k, dw_q=sums[0], dw_k=sums[1])
    assert all(torch.equal(a, b) for a, b in zip(got, want[2:])) and all(torch.equal(gap, how(c)[name]) for name, gap in gaps.items())

def test_qk_norm_rope_binding_refuses_other_types_and_layouts():
    b = lambda *s, t=BF16: torch.zeros(s, dtype=t)
    freq, pos = torch.zeros(8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        rl.relibra_qk_norm_rope_fwd(b(4, 2, 16, t=torch.float32), b(4, 1, 16), pos, freq)
    with pytest.raises(AssertionError):
        rl.relibra_qk_norm_rope_fwd(b(4, 2, 16), b(4, 1, 16), pos.long(), freq)
    with pytest.raises(AssertionError):
        rl.relibra_qk_norm_rope_fwd(b(4, 2, 16), b(4, 1, 16), pos, None)
    with pytest.raises(AssertionError):
        rl.relibra_qk_norm_rope_fwd(b(4, 2, 16), b(4, 1, 16), pos, freq, axis=[0] * 7)
    with pytest.raises(AssertionError):
        rl.relibra_qk_norm_rope_fwd(b(4, 16, 2).transpose(1, 2), b(4, 1, 16), pos, freq)
