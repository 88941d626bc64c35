"""Router gates of replayed ids, the balance loss over per-expert counts, and their gradients: against plain double precision.

Tolerances.  A score is exp(v - m) of fp32 inputs: the difference is rounded once (2^-24 of at most `spread`, which exp turns into
a relative error), exp, the reciprocal and the products add a few roundings, a sum over a row at most log2(E) + 8 more in the
order it is taken.  ROUNDINGS = 48 such steps of 2^-24 cover it; differences (gradients) are held against the size of
their terms.  A result stored in bf16 is off by another half step, 2^-8 of its value."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
U32 = torch.finfo(torch.float32).eps / 2
ROUNDINGS = 48


def make(n_mb, T, E, k, dtype=torch.float32, seed=0, spread=3.0, padded=False, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    z = spread * torch.randn((n_mb, T, E), generator=g)
    if masked:
        z[torch.rand((n_mb, T, E), generator=g) < masked] = -math.inf
    ids = torch.argsort(torch.rand((n_mb, T, E), generator=g), dim=2)[:, :, :k].to(torch.int32).contiguous()
    valid = (torch.rand((n_mb, T), generator=g) < 0.6).to(torch.uint8) if padded else None
    return z.to(dtype), ids, valid


def definition(z, ids, valid, sigmoid, normalize, scale, coef):
    """gates, counts, n_valid, prob_mean, loss in double, differentiable in z; ids outside [0, E) give nothing."""
    n_mb, T, E = z.shape
    k = ids.shape[2]
    live = torch.ones((n_mb, T), dtype=torch.bool) if valid is None else valid != 0
    z = torch.where(live[..., None], z, torch.zeros_like(z))
    u = torch.nn.functional.logsigmoid(z) if sigmoid else z

    def softmax(v, dim):
        top = v.detach().amax(dim, keepdim=True)
        e = torch.exp(v - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        e = torch.where(v == -math.inf, torch.zeros_like(e), e)
        s = e.sum(dim, keepdim=True)
        return e / torch.where(s > 0, s, torch.ones_like(s))

    p = softmax(u, 2)
    inside = (ids >= 0) & (ids < E)
    at = ids.clamp(0, E - 1).long()
    us = torch.where(inside, u.gather(2, at), torch.full((), -math.inf, dtype=u.dtype))
    if normalize:
        part = softmax(us, 2)
    else:
        part = (torch.sigmoid(z) if sigmoid else p).gather(2, at) * inside
    counts = torch.zeros((n_mb, E), dtype=torch.int64)
    for s in range(k):
        counts.scatter_add_(1, at[:, :, s], (inside[:, :, s] & live).long())
    n = live.sum(1)
    nn = n.clamp(min=1).double()
    mean = (p * live[..., None]).sum(1) / nn[:, None]
    loss = coef * E * (counts.double() / (k * nn[:, None]) * mean).sum(1) * (n > 0)
    return scale * part * live[..., None], counts, n, mean, loss


def spread_of(z):
    f = z[torch.isfinite(z)].double()
    return float(f.max() - f.min()) if f.numel() else 0.0


CASES = [
    # n_mb, T, E, k: one token; one expert; rows of every layout, divisible by 8 and not; more selections than lanes; a wide router
    dict(n_mb=1, T=1, E=128, k=8), dict(n_mb=1, T=1, E=1, k=1), dict(n_mb=2, T=65, E=8, k=8), dict(n_mb=3, T=77, E=7, k=3), dict(n_mb=1, T=130, E=16, k=11),
    dict(n_mb=2, T=33, E=60, k=6), dict(n_mb=1, T=300, E=128, k=8), dict(n_mb=2, T=19, E=255, k=16), dict(n_mb=1, T=9, E=512, k=64), dict(n_mb=1, T=13, E=1000, k=5),
    dict(n_mb=1, T=5, E=2048, k=8), dict(n_mb=1, T=6, E=4096, k=64), dict(n_mb=40, T=3, E=32, k=4), dict(n_mb=1, T=5000, E=24, k=2),
]


@gpu
@pytest.mark.parametrize("score", [(False, True), (False, False), (True, True), (True, False)], ids=["softmax-norm", "softmax", "sigmoid-norm", "sigmoid"])
@pytest.mark.parametrize("kw", CASES, ids=lambda c: "x".join(str(v) for v in c.values()))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_router_against_the_definition(kw, score, dtype):
    sigmoid, normalize = score
    check(kw, sigmoid, normalize, dtype, padded=kw["T"] > 4, masked=0.2)


def check(kw, sigmoid, normalize, dtype, padded, masked, seed=0, spread=3.0, z=None, ids=None, valid=None, flag=0):
    n_mb, T, E, k = kw["n_mb"], kw["T"], kw["E"], kw["k"]
    if z is None:
        z, ids, valid = make(n_mb, T, E, k, dtype, seed, spread, padded, masked)
    scale, coef = 2.5, 0.01
    dg = torch.randn((n_mb, T, k), generator=torch.Generator().manual_seed(seed + 1))
    dl = 1000.0 * torch.rand(n_mb, generator=torch.Generator().manual_seed(seed + 2))
    zd = z.double().requires_grad_(True)
    want = definition(zd, ids, valid, sigmoid, normalize, scale, coef)
    ((want[0] * dg.double()).sum() + (want[4] * dl.double()).sum()).backward()
    dev = lambda t: None if t is None else t.to(DEV)
    err = rl.new_err_flag()
    how = dict(sigmoid=sigmoid, normalize=normalize, scale=scale, balance_coef=coef, valid=dev(valid), err_flag=err)
    got = rl.relibra_router_fwd(dev(z), dev(ids), **how)
    dz = rl.relibra_router_bwd(dev(z), dev(ids), dev(dg), got[1], got[2], dev(dl), **how)
    assert err.item() == flag
    rel = (ROUNDINGS + spread_of(z)) * U32
    assert torch.equal(got[1].cpu().long(), want[1]) and torch.equal(got[2].cpu().long(), want[2])
    for g, w in ((got[0], want[0]), (got[3], want[3]), (got[4], want[4])):
        w = w.detach()
        assert torch.all((g.cpu().double() - w).abs() <= rel * w.abs() + 1e-37), float((g.cpu().double() - w).abs().max())
    # the gradient's terms: p (|d| + sum p |d|) of the loss (and of plain softmax gates), part (|dg| + sum part |dg|) of the gates
    with torch.no_grad():
        live = torch.ones((n_mb, T), dtype=torch.float64) if valid is None else (valid != 0).double()
        p = definition(zd, ids, None, sigmoid, normalize, 1.0, 1.0)
        part = p[0].abs()
        u = torch.nn.functional.logsigmoid(zd) if sigmoid else zd
        prob = torch.softmax(torch.where(torch.isneginf(u.amax(2, keepdim=True)), torch.zeros_like(u), u), 2).nan_to_num()
        n = want[2].clamp(min=1).double()[:, None]
        cost = dl.double()[:, None] * coef * E * want[1].double() / (k * n * n)
        inside = (ids >= 0) & (ids < E)
        put = torch.zeros_like(prob).scatter_add_(2, ids.clamp(0, E - 1).long(), (scale * dg.double()).abs() * inside * (1 if not normalize and not sigmoid else part + (part if normalize else 0) * 1))
        mag = prob * (cost[:, None, :] + (prob * cost[:, None, :]).sum(2, keepdim=True))
        if normalize or sigmoid:
            mag = mag + put + (part * (scale * dg.double()).abs()).sum(2, keepdim=True) * torch.zeros_like(prob).scatter_add_(2, ids.clamp(0, E - 1).long(), part * inside)
        else:
            mag = mag + prob * (put + (prob * put).sum(2, keepdim=True))
        mag = mag * live[..., None]
    half = torch.finfo(dtype).eps / 2
    w = zd.grad.nan_to_num()
    off = (dz.cpu().double() - w).abs()
    assert torch.all(off <= half * w.abs() + 2 * rel * mag + 1e-37), (float(off.max()), float((off - half * w.abs() - 2 * rel * mag).max()))
    return got, dz


@gpu
def test_router_long_micro_batches_give_the_same_every_time():
    """Many rounds of tokens in every block, its waves running apart, over several passes."""
    kw = dict(n_mb=12, T=6000, E=128, k=8)
    got, dz = check(kw, False, True, torch.bfloat16, True, 0.0, seed=31)
    z, ids, valid = make(12, 6000, 128, 8, torch.bfloat16, 31, 3.0, True, 0.0)
    for _ in range(10):
        again = rl.relibra_router_fwd(z.to(DEV), ids.to(DEV), scale=2.5, balance_coef=0.01, valid=valid.to(DEV))
        assert all(torch.equal(a, b) for a, b in zip(again, got))


@gpu
def test_router_gradient_against_differences():
    """Central differences of the library's own forward pass: loss and gates as functions of single logits."""
    n_mb, T, E, k = 1, 4, 12, 3
    z, ids, _ = make(n_mb, T, E, k, seed=5, spread=1.0)
    dg = torch.randn((n_mb, T, k), generator=torch.Generator().manual_seed(6))
    for sigmoid, normalize in ((False, True), (True, True), (False, False), (True, False)):
        how = dict(sigmoid=sigmoid, normalize=normalize, scale=1.0, balance_coef=1.0)
        zd, idd = z.to(DEV), ids.to(DEV)
        f = rl.relibra_router_fwd(zd, idd, **how)
        grad = rl.relibra_router_bwd(zd, idd, dg.to(DEV), f[1], f[2], torch.ones(1, device=DEV), **how).cpu().double()
        value = lambda zz: (lambda o: float((o[0].cpu().double() * dg.double()).sum() + o[4].cpu().double().sum()))(rl.relibra_router_fwd(zz, idd, **how))
        step = 2.0 ** -6
        for t in range(T):
            for e in range(E):
                up, dn = zd.clone(), zd.clone()
                up[0, t, e] += step
                dn[0, t, e] -= step
                diff = (value(up) - value(dn)) / float(up[0, t, e] - dn[0, t, e])
                # third derivative: at most about 1 per unit of |dg| and loss: step^2 / 6 * 10; rounding of the values: 40 * 2^-24 / step
                assert abs(diff - float(grad[0, t, e])) <= 10 * step * step / 6 + 40 * U32 / step


@gpu
def test_router_masks_that_leave_nothing_and_far_selections():
    """Rows of -infinities, selected experts all masked, and selected logits far below the row's largest."""
    E, k = 16, 4
    z = torch.zeros((1, 6, E))
    z[0, 0] = -math.inf                                      # nothing in the row
    z[0, 1, :4] = -math.inf                                  # nothing among the selected
    z[0, 2, 4] = 300.0                                       # the selected far below the row's largest
    z[0, 3] = -200.0                                         # every sigmoid underflows
    z[0, 4, :2] = -math.inf
    z[0, 5] = torch.finfo(torch.float32).min                 # the lowest value everywhere is no mask: an even row
    ids = torch.arange(k, dtype=torch.int32).expand(1, 6, k).contiguous()
    for sigmoid in (False, True):
        err = rl.new_err_flag()
        gates, counts, n, mean, loss = rl.relibra_router_fwd(z.to(DEV), ids.to(DEV), sigmoid=sigmoid, normalize=True, balance_coef=1.0, err_flag=err)
        g = gates.cpu()[0]
        assert torch.all(g[0] == 0) and torch.all(g[1] == 0)
        assert torch.allclose(g[2], torch.full((k,), 0.25)) and torch.allclose(g[3], torch.full((k,), 0.25)) and torch.allclose(g[4], torch.tensor([0.0, 0.0, 0.5, 0.5]))
        assert torch.allclose(g[5], torch.full((k,), 0.25))
        assert counts.cpu()[0, :4].tolist() == [6] * 4 and n.item() == 6 and torch.isfinite(mean).all() and torch.isfinite(loss).all() and err.item() == 0
        dz = rl.relibra_router_bwd(z.to(DEV), ids.to(DEV), torch.ones_like(gates), counts, n, torch.ones(1, device=DEV), sigmoid=sigmoid, balance_coef=1.0)
        assert torch.isfinite(dz).all() and torch.all(dz[0, 0] == 0)


@gpu
def test_router_padding_is_not_looked_at_and_nan_stays_with_its_token():
    E, k = 32, 4
    z, ids, _ = make(2, 50, E, k, seed=9)
    valid = torch.ones((2, 50), dtype=torch.bool)
    valid[0, 40:] = False
    valid[1, :] = False                                      # a micro-batch of padding only
    want = [t.cpu() for t in rl.relibra_router_fwd(z.to(DEV), ids.to(DEV), valid=valid.to(DEV), balance_coef=1.0)]
    zz, ii = z.clone(), ids.clone()
    zz[0, 40:] = math.nan
    zz[1] = math.inf
    ii[0, 45:] = 1 << 30
    ii[1] = -5
    err = rl.new_err_flag()
    got = rl.relibra_router_fwd(zz.to(DEV), ii.to(DEV), valid=valid.to(DEV), balance_coef=1.0, err_flag=err)
    assert err.item() == 0 and all(torch.equal(a.cpu(), b) for a, b in zip(got, want))
    assert got[2].tolist() == [40, 0] and got[4][1].item() == 0 and torch.all(got[3][1] == 0) and torch.all(got[0][0, 40:] == 0)
    dz = rl.relibra_router_bwd(zz.to(DEV), ii.to(DEV), torch.ones_like(got[0]), got[1], got[2], torch.ones(2, device=DEV), valid=valid.to(DEV), balance_coef=1.0, err_flag=err)
    assert err.item() == 0 and torch.all(dz[0, 40:] == 0) and torch.all(dz[1] == 0) and torch.isfinite(dz).all()
    zz = z.clone()
    zz[0, 3, 5] = math.nan
    gates, _, _, mean, loss = rl.relibra_router_fwd(zz.to(DEV), ids.to(DEV), normalize=False, balance_coef=1.0)
    bad = torch.isnan(gates.cpu()).any(2)
    assert bad[0, 3] and bad.sum() == 1 and torch.isnan(loss[0]) and torch.isfinite(loss[1])


@gpu
@pytest.mark.parametrize("normalize", [True, False])
def test_router_bad_ids_and_the_same_expert_twice(normalize):
    E, k = 20, 5
    z, ids, _ = make(2, 70, E, k, seed=3)
    ids[0, 5, 1], ids[0, 6, 0], ids[1, 0, :] = E, -1, 99
    ids[0, 8, :] = 7                                         # one expert in all places
    ids[1, 9, 1:] = ids[1, 9, :1]
    check(dict(n_mb=2, T=70, E=E, k=k), False, normalize, torch.float32, False, 0.0, z=z, ids=ids, flag=rl.ERR_ID_RANGE)


@gpu
def test_router_sizes_of_zero():
    z, ids = torch.zeros((3, 0, 8), device=DEV), torch.zeros((3, 0, 2), dtype=torch.int32, device=DEV)
    gates, counts, n, mean, loss = rl.relibra_router_fwd(z, ids, balance_coef=1.0)
    assert gates.shape == (3, 0, 2) and counts.abs().sum() == 0 and n.sum() == 0 and mean.sum() == 0 and loss.sum() == 0
    assert rl.relibra_router_bwd(z, ids, gates, counts, n, loss).shape == (3, 0, 8)
    got = rl.relibra_router_fwd(torch.zeros((0, 4, 8), device=DEV), torch.zeros((0, 4, 2), dtype=torch.int32, device=DEV))
    assert got[0].shape == (0, 4, 2) and got[4].shape == (0,)


@gpu
def test_router_gates_feed_the_path_and_only_parts_of_the_gradient():
    """Without dloss the gradient is the gates' alone, without dgates the loss's alone, and the two add up."""
    z, ids, valid = make(2, 90, 64, 6, seed=11, padded=True)
    zd, idd, vd = z.to(DEV), ids.to(DEV), valid.to(DEV)
    f = rl.relibra_router_fwd(zd, idd, valid=vd, balance_coef=2.0)
    dg, dl = torch.randn_like(f[0]), torch.full((2,), 50.0, device=DEV)
    both = rl.relibra_router_bwd(zd, idd, dg, f[1], f[2], dl, valid=vd, balance_coef=2.0)
    gate = rl.relibra_router_bwd(zd, idd, dg, valid=vd, balance_coef=2.0)
    bal = rl.relibra_router_bwd(zd, idd, None, f[1], f[2], dl, valid=vd, balance_coef=2.0)
    assert (both - gate - bal).abs().max().item() <= 4 * U32 * (gate.abs().max() + bal.abs().max()).item()


@gpu
def test_router_in_a_graph_beside_eager_calls():
    """Captured with its own buffers, replayed between eager calls on other inputs and on another stream; every replay equals the eager result."""
    z, ids, valid = make(4, 257, 128, 8, torch.bfloat16, seed=21, padded=True)
    zd, idd, vd = z.to(DEV), ids.to(DEV), valid.to(DEV)
    err = rl.new_err_flag()
    ws = rl.router_workspace(4, 257, 8, 128)
    dl = torch.full((4,), 100.0, device=DEV)
    dg = torch.randn((4, 257, 8), device=DEV)

    def step(zz, **kw):
        f = rl.relibra_router_fwd(zz, idd, valid=vd, balance_coef=1.0, err_flag=err, **kw)
        return (*f, rl.relibra_router_bwd(zz, idd, dg, f[1], f[2], dl, valid=vd, balance_coef=1.0, err_flag=err))
    step(zd, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    src = zd.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(src, workspace=ws)
    side = torch.cuda.Stream()
    for turn in range(3):
        src.copy_(zd * (1 + turn))
        want = step(src.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step(src)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), turn
    assert err.item() == 0


# ------------------------------------------------------------------ refusals (no GPU needed: nothing is launched)
def _fwd(n_mb=1, T=4, k=2, E=8, flags=2, logits=4096, ids=4096, gates=4096, counts=4096, ws=4096, ws_bytes=1 << 30, err=4096):
    p = C.c_void_p
    return rl.lib().relibra_router_fwd(p(logits), p(ids), p(0), n_mb, T, k, E, flags, C.c_float(1), C.c_float(1), p(gates), p(counts), p(4096), p(4096), p(4096),
                                       p(ws), C.c_size_t(ws_bytes), p(err), p(0))


def _bwd(n_mb=1, T=4, k=2, E=8, flags=2, logits=4096, ids=4096, counts=4096, n_valid=4096, dloss=4096, dlogits=4096, err=4096):
    p = C.c_void_p
    return rl.lib().relibra_router_bwd(p(logits), p(ids), p(0), p(4096), p(counts), p(n_valid), p(dloss), n_mb, T, k, E, flags, C.c_float(1), C.c_float(1),
                                       p(dlogits), p(err), p(0))


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_router_refusals(call):
    for bad in (dict(n_mb=-1), dict(T=-1), dict(E=0), dict(k=0), dict(k=9), dict(flags=8), dict(logits=0), dict(ids=0), dict(logits=4104), dict(err=0)):
        assert call(**bad) == rl.EINVAL, bad
    for bad in (dict(E=4097), dict(E=100, k=65), dict(n_mb=65536), dict(n_mb=4, T=1 << 29)):
        assert call(**bad) == rl.EUNSUPPORTED, bad
    assert call(n_mb=0) == rl.OK


def test_router_refuses_missing_outputs_and_small_workspaces():
    assert _fwd(gates=0) == rl.EINVAL and _fwd(counts=0) == rl.EINVAL
    need = rl.workspace_bytes(rl.WS_ROUTER, 4, 2, 8, 1, 0, 0)
    assert need > 0 and _fwd(ws_bytes=need - 1) == rl.EWORKSPACE and _fwd(ws=0) == rl.EWORKSPACE and _fwd(ws=4104) == rl.EINVAL
    assert _bwd(dlogits=0) == rl.EINVAL and _bwd(counts=0) == rl.EINVAL and _bwd(n_valid=0) == rl.EINVAL and _bwd(T=0) == rl.OK
    assert rl.workspace_bytes(rl.WS_ROUTER, 1 << 29, 1, 8, 4, 0, 0) == 0


@gpu
@pytest.mark.parametrize("kw", [dict(n_mb=1, T=9000, E=1000, k=4), dict(n_mb=2, T=4099, E=256, k=8), dict(n_mb=1, T=1200, E=4096, k=16), dict(n_mb=1, T=20000, E=128, k=8)],
                         ids=lambda c: "x".join(str(v) for v in c.values()))
def test_router_few_long_micro_batches(kw):
    """So many blocks that their sums are folded before they are finished.  A value passes at most 4 + 5 additions in a block, 9 in a
    wave of a fold, 3 between the waves and 16 behind them: fewer than ROUNDINGS with the score's own."""
    check(kw, False, True, torch.bfloat16, True, 0.1, seed=77)


class _Elsewhere:
    """A contiguous tensor of device 1."""
    dtype = torch.float32

    def get_device(self):
        return 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(rl, "_device", lambda: 0)
    with pytest.raises(AssertionError, match="current device"):
        rl._ptrs(_Elsewhere())
    monkeypatch.setattr(rl, "_device", lambda: 1)
    assert rl._ptrs(None, _Elsewhere()) == [None, 4096]
    with pytest.raises(AssertionError, match="contiguous"):
        rl._ptrs(torch.zeros(4))


def test_router_refuses_more_selections_than_a_count_holds():
    assert _fwd(T=1 << 28, k=8) == rl.EUNSUPPORTED and _bwd(T=1 << 28, k=8) == rl.EUNSUPPORTED
    assert rl.workspace_bytes(rl.WS_ROUTER, 4, 2, 4097, 1, 0, 0) == 0 and rl.workspace_bytes(rl.WS_ROUTER, 4, 2, 8, 65536, 0, 0) == 0


@gpu
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_router_positive_infinity(dtype, normalize):
    """A sigmoid of +infinity is 1, as that of 200 in fp32: every result is the same bit for bit.  A softmax is NaN there, and stays with its token
    and its micro-batch's means; gates normalised over other selections are not touched."""
    E, k = 24, 3
    z, ids, _ = make(2, 40, E, k, dtype, seed=41)
    z[0, 4, 6] = z[0, 5, ids[0, 5, 1]] = 200.0
    ids[0, 4] = torch.tensor([0, 1, 2], dtype=torch.int32)   # the infinite logit is not selected here
    zi = z.clone()
    zi[z == 200.0] = math.inf
    dg, dl = torch.randn((2, 40, k), device=DEV), torch.full((2,), 30.0, device=DEV)

    def both(zz, sigmoid):
        how = dict(sigmoid=sigmoid, normalize=normalize, balance_coef=1.0)
        f = rl.relibra_router_fwd(zz.to(DEV), ids.to(DEV), **how)
        return (*f, rl.relibra_router_bwd(zz.to(DEV), ids.to(DEV), dg, f[1], f[2], dl, **how))
    a, b = both(zi, True), both(z, True)
    assert all(torch.isfinite(x.float()).all() and torch.equal(x, y) for x, y in zip(a, b))
    a, b = both(zi, False), both(z, False)
    hit = torch.zeros((2, 40), dtype=torch.bool)
    hit[0, 4:6] = True
    assert torch.isnan(a[3][0]).all() and torch.isnan(a[4][0]) and torch.equal(a[3][1], b[3][1]) and torch.equal(a[4][1], b[4][1])
    assert torch.equal(a[0][~hit], b[0][~hit]) and torch.equal(a[5][~hit], b[5][~hit]) and torch.isnan(a[0][0, 5]).any()
    assert torch.isnan(a[5][0, 4:6].float()).all() and (torch.equal(a[0][0, 4], b[0][0, 4]) if normalize else torch.isnan(a[0][0, 4]).all())


@gpu
@pytest.mark.parametrize("kw", [dict(n_mb=1, T=1, E=1, k=1), dict(n_mb=3, T=77, E=7, k=3), dict(n_mb=2, T=301, E=60, k=6), dict(n_mb=1, T=9000, E=1000, k=4), dict(n_mb=2, T=513, E=255, k=40)],
                         ids=lambda c: "x".join(str(v) for v in c.values()))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_router_writes_every_value_and_nothing_else(kw, dtype):
    """Outputs and workspace of NaN bits before the calls, NaN bits around them."""
    n_mb, T, E, k = kw["n_mb"], kw["T"], kw["E"], kw["k"]
    z, ids, valid = make(n_mb, T, E, k, dtype, seed=51, padded=T > 4)
    how = dict(sigmoid=True, valid=None if valid is None else valid.to(DEV), balance_coef=0.5)
    zd, idd, dg, dl = z.to(DEV), ids.to(DEV), torch.randn((n_mb, T, k), device=DEV), torch.full((n_mb,), 9.0, device=DEV)
    want = rl.relibra_router_fwd(zd, idd, **how)
    want_dz = rl.relibra_router_bwd(zd, idd, dg, want[1], want[2], dl, **how)
    kept = []

    def full(shape, t, pad=64):
        count = math.prod(shape)
        flat = torch.full((count + 2 * pad,), 255 if t.itemsize == 1 else -1, dtype={1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.itemsize], device=DEV)
        kept.append(lambda: bool((torch.cat([flat[:pad], flat[pad + count:]]) == (255 if t.itemsize == 1 else -1)).all()))
        return flat.view(t)[pad:pad + count].view(shape)
    out = dict(gates=full((n_mb, T, k), torch.float32), counts=full((n_mb, E), torch.int32), n_valid=full((n_mb,), torch.int32), prob_mean=full((n_mb, E), torch.float32),
               loss=full((n_mb,), torch.float32))
    ws = full((rl.workspace_bytes(rl.WS_ROUTER, T, k, E, n_mb, 0, 0),), torch.uint8, 256)
    got = rl.relibra_router_fwd(zd, idd, **how, **out, workspace=ws)
    dz = rl.relibra_router_bwd(zd, idd, dg, got[1], got[2], dl, **how, dlogits=full((n_mb, T, E), dtype))
    assert all(torch.equal(a, b) for a, b in zip((*got, dz), (*want, want_dz))) and torch.isfinite(dz.float()).all()
    assert all(k() for k in kept)
