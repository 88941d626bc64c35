"""One training step of a whole MoE block through the library: norm, router gates of replayed ids with the balance loss, dispatch,
expert FFN, combine, norm and residual; back through all of it; then the orthogonalised update of the experts.  Against torch's
differentiation of the same block in double precision.

Tolerance: between the input and any gradient lie at most 14 roundings to bf16 one behind the other (n, Gt, U, A, rows, y, x', n' forward;
the upstream rows, dGt, dU, dx rows, their sum, dx backward), each 2^-8 / sqrt(12) * 1.5 = 1.7e-3 of the norm in the root mean
square: sqrt(14) * 1.7e-3 = 6.4e-3.  TOL = 1.2e-2 leaves a factor of two for what the products magnify."""
import numpy as np
import pytest
import torch

import workloads as wl
import paper_2605_08639_amd as rl

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOL = 1.2e-2
EPS, RHO, COEF = 1e-5, 0.8, 0.02


def rms(v, w):
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w


def reference(p, ids, T, k, E, up_x, up_n, sigmoid):
    """The block in double; p: dict of leaf tensors."""
    n = rms(p["x"], p["w1"])
    z = n @ p["Wr"].T
    u = torch.nn.functional.logsigmoid(z) if sigmoid else z
    prob = torch.softmax(u, 1)
    gates = torch.softmax(u.gather(1, ids), 1)
    counts = torch.bincount(ids.reshape(-1), minlength=E).double()
    loss = COEF * E * (counts / (k * T) * prob.mean(0)).sum()
    y = torch.zeros_like(n)
    for e in range(E):
        t, s = torch.nonzero(ids == e, as_tuple=True)
        if t.numel():
            rows = n[t]
            a = torch.nn.functional.silu(rows @ p["Wg"][e].T) * (rows @ p["Wu"][e].T)
            y = y.index_add(0, t, gates[t, s][:, None] * (a @ p["Wd"][e].T))
    x_out = RHO * p["x"] + p["g"][:, None] * rms(y, p["w2"])
    n_out = rms(x_out, p["w3"])
    return x_out, n_out, loss, counts, (x_out * up_x).sum() + (n_out * up_n).sum() + 500.0 * loss


@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
def test_training_step_of_a_block(sigmoid):
    cfg = wl.small_config(E=16, k=4, h=256, hff=192, T=333, EP=4, r=2, n_mb=1)
    E, k, h, hff, T = cfg.E, cfg.k, cfg.h, cfg.hff, cfg.T
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=gen)
    b = lambda t: t.to(torch.bfloat16)
    p = dict(x=b(r(T, h)), w1=b(1 + 0.2 * r(h)), w2=b(1 + 0.2 * r(h)), w3=b(1 + 0.2 * r(h)), Wr=b(0.15 * r(E, h)), Wg=b(0.06 * r(E, hff, h)), Wu=b(0.06 * r(E, hff, h)),
             Wd=b(0.06 * r(E, h, hff)), g=torch.sigmoid(r(T)))
    up_x, up_n = b(r(T, h)), b(r(T, h))
    d = {name: t.to(DEV) for name, t in p.items()}
    err = rl.new_err_flag()

    # ---- forward
    _, n = rl.relibra_block_norm_fwd(d["x"], w_pre=d["w1"], eps=EPS)
    logits = n.float() @ d["Wr"].float().T                   # the router's own product is the program's
    ids = torch.topk(logits.cpu() + 0.3 * r(T, E), k, dim=1).indices.to(torch.int32)        # replayed: not quite these logits'
    ids_d = ids.to(DEV)
    how = dict(sigmoid=sigmoid, normalize=True, balance_coef=COEF, err_flag=err)
    gates, counts, n_valid, _, loss = rl.relibra_router_fwd(logits[None], ids_d[None], **how)
    assert torch.equal(counts, rl.relibra_route_hist(ids_d[None], E)) and n_valid.item() == T
    plan = rl.relibra_plan(counts.cpu().numpy(), k, cfg.EP, cfg.rpn, cfg.r)
    tab = {key: torch.from_numpy(np.ascontiguousarray(plan[key][0])).to(DEV) for key in ("inst_ptr", "inst_rows", "inst_group", "group_offset", "group_expert", "group_dw_slot")}
    row_of, _, rows = rl.relibra_permute(ids_d, tab["inst_ptr"], tab["inst_rows"], tab["inst_group"], tab["group_offset"], n, E, cfg.G, err_flag=err)
    Gt, U, A, Y = rl.relibra_moe_ffn_fwd(rows, tab["group_offset"], tab["group_expert"], d["Wg"], d["Wu"], d["Wd"], err_flag=err)
    y = rl.relibra_unpermute_combine(rl.COMBINE_FWD, Y, row_of, T, k, gates=gates[0], err_flag=err)
    x_out, n_out = rl.relibra_block_norm_fwd(d["x"], y=y, w_post=d["w2"], w_pre=d["w3"], gate=d["g"], res_scale=RHO, eps=EPS)

    # ---- backward
    dx, dy, dg, dw2, dw3 = rl.relibra_block_norm_bwd(x_out, up_x.to(DEV), up_n.to(DEV), y=y, w_post=d["w2"], w_pre=d["w3"], gate=d["g"], res_scale=RHO, eps=EPS)
    dY, dgates = rl.relibra_unpermute_combine(rl.COMBINE_BWD, Y, row_of, T, k, gates=gates[0], tok=dy, err_flag=err)
    slots = E + cfg.EP * cfg.r
    dWg, dWu, dWd = (torch.empty(s, device=DEV) for s in ((slots, hff, h), (slots, hff, h), (slots, h, hff)))
    drows = rl.relibra_moe_ffn_bwd(dY, rows, Gt, U, A, tab["group_offset"], tab["group_expert"], tab["group_dw_slot"], d["Wg"], d["Wu"], d["Wd"], dWg, dWu, dWd, err_flag=err)
    dn = rl.relibra_unpermute_combine(rl.COMBINE_SUM, drows, row_of, T, k, err_flag=err)
    dlogits = rl.relibra_router_bwd(logits[None], ids_d[None], dgates[None], counts, n_valid, torch.full((1,), 500.0, device=DEV), **how)[0]
    dWr = dlogits.T @ n.float()
    dn = (dn.float() + dlogits @ d["Wr"].float()).to(torch.bfloat16)
    dx, _, _, _, dw1 = rl.relibra_block_norm_bwd(d["x"], dx, dn, w_pre=d["w1"], eps=EPS)
    torch.cuda.synchronize()
    assert err.item() == 0

    # ---- the same in double
    q = {name: t.double().requires_grad_(True) for name, t in p.items()}
    want_x, want_n, want_loss, want_counts, goal = reference(q, ids.long(), T, k, E, up_x.double(), up_n.double(), sigmoid)
    goal.backward()
    rel = lambda a, w: float((a.cpu().double() - w.detach()).norm() / w.detach().norm())
    errs = dict(x_out=rel(x_out, want_x), n_out=rel(n_out, want_n), loss=rel(loss[0], want_loss), dx=rel(dx, q["x"].grad), dw1=rel(dw1, q["w1"].grad), dw2=rel(dw2, q["w2"].grad),
                dw3=rel(dw3, q["w3"].grad), dg=rel(dg, q["g"].grad), dWr=rel(dWr, q["Wr"].grad), dWg=rel(dWg[:E], q["Wg"].grad), dWu=rel(dWu[:E], q["Wu"].grad), dWd=rel(dWd[:E], q["Wd"].grad))
    assert torch.equal(counts[0].cpu().double(), want_counts)
    assert max(errs.values()) <= TOL, errs

    # ---- the update, from the gradients as they lie in the slot arrays
    for grad, weight in ((dWg[:E], d["Wg"]), (dWu[:E], d["Wu"]), (dWd[:E], d["Wd"])):
        out, mom = rl.relibra_orthogonalize(grad, momentum=torch.zeros_like(grad), mu=0.9, nesterov=True, scale=0.2 * max(grad.shape[1:]) ** 0.5)
        assert torch.equal(mom, grad)
        new = weight - (1e-3 * out).to(torch.bfloat16)
        assert torch.isfinite(new.float()).all()
        for e in range(E):
            top = torch.linalg.svdvals(out[e].cpu().double()) / (0.2 * max(grad.shape[1:]) ** 0.5)
            assert top[0] < 1.25 and (want_counts[e] == 0 or top[0] > 0.65)      # the five steps take every leading value there
