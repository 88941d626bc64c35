"""The attention half of a block in a training step through the library: norm, fused projection, norms and rotation of queries and keys, attention of
packed and padded sequences, output projection, norm and residual; back through all of it.  Against torch's differentiation of the same in
double precision.

Tolerance: between the input and any gradient lie at most 12 roundings to bf16 one behind the other (n, qkv, q' and k', p, out, o, n' forward; dy, dout, p and ds,
dqkv, its rotation, dn, dx backward), each 2^-8 / sqrt(12) * 1.5 = 1.7e-3 of the norm in the root mean square: sqrt(12) * 1.7e-3 = 5.9e-3.  TOL = 1.2e-2 leaves a
factor of two for what products and the softmax magnify."""
import math

import pytest
import torch

import paper_2605_08639_amd as rl

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOL = 1.2e-2
EPS, RHO = 1e-5, 0.8
BF16 = torch.bfloat16


def rms(v, w):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * w


def rotate(x, angle):
    half = angle.shape[1]
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    return torch.cat([a * c - b * s, b * c + a * s, rest], -1)


def reference(p, angle, seqs, Hq, Hk, d, up_x, up_n):
    T = p["x"].shape[0]
    n = rms(p["x"], p["w1"])
    q, k, v = (t.unflatten(1, (-1, d)) for t in torch.split(n @ p["Wqkv"].T, [Hq * d, Hk * d, Hk * d], dim=1))
    q, k = rotate(rms(q, p["wq"]), angle), rotate(rms(k, p["wk"]), angle)
    out = torch.zeros((T, Hq, d), dtype=torch.float64)
    for a, n_tok in seqs:
        rows = slice(a, a + n_tok)
        kk, vv = (t[rows].repeat_interleave(Hq // Hk, 1).transpose(0, 1) for t in (k, v))
        z = (q[rows].transpose(0, 1) @ kk.transpose(1, 2)) / math.sqrt(d)
        z = z.masked_fill(torch.ones(n_tok, n_tok, dtype=torch.bool).triu(1), -math.inf)
        out = out.index_add(0, torch.arange(a, a + n_tok), (torch.softmax(z, 2) @ vv).transpose(0, 1))
    o = out.flatten(1) @ p["Wo"].T
    x_out = RHO * p["x"] + rms(o, p["w2"]) * p["g"][:, None]
    n_out = rms(x_out, p["w3"])
    return x_out, n_out, (x_out * up_x).sum() + (n_out * up_n).sum()


@pytest.mark.parametrize("axes", [1, 3], ids=["text", "images"])
def test_training_step_of_attention(axes):
    Hq, Hk, d, h, rot = 6, 2, 64, 256, 32 if axes == 1 else 64
    starts, lens = [0, 150, 290, 333], [150, 131, 43]
    T, width = 333, (Hq + 2 * Hk) * d
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen)
    b = lambda t: t.to(BF16)
    p = dict(x=b(r(T, h)), w1=b(1 + 0.2 * r(h)), w2=b(1 + 0.2 * r(h)), w3=b(1 + 0.2 * r(h)), Wqkv=b(r(width, h) / math.sqrt(h)), Wo=b(r(h, Hq * d) / math.sqrt(Hq * d)), wq=b(1.5 + 0.2 * r(d)),
             wk=b(1 + 0.2 * r(d)), g=torch.sigmoid(r(T)))
    freq = (1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float()
    pos = torch.randint(0, 400, (axes, T), generator=gen, dtype=torch.int32)
    axis = None if axes == 1 else [j * 3 // (rot // 2) for j in range(rot // 2)]
    real = torch.zeros(T)
    for a, n_tok in zip(starts, lens):
        real[a:a + n_tok] = 1
    up_x, up_n = b(r(T, h) * real[:, None]), b(r(T, h) * real[:, None])          # padding has no upstream
    D = {name: t.to(DEV) for name, t in p.items()}
    start, length = torch.tensor(starts, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    turn = dict(pos=pos.to(DEV), freq=freq.to(DEV), w_q=D["wq"], w_k=D["wk"], axis=axis, eps=EPS)
    flag = rl.new_err_flag()
    parts = lambda whole: [t.unflatten(1, (-1, d)) for t in torch.split(whole, [Hq * d, Hk * d, Hk * d], dim=1)]

    # ---- forward
    _, n = rl.relibra_block_norm_fwd(D["x"], w_pre=D["w1"], eps=EPS)
    qkv = n @ D["Wqkv"].T                                    # projections are the program's
    q, k, v = parts(qkv)
    q1, k1 = rl.relibra_qk_norm_rope_fwd(q, k, **turn)
    out, lse = rl.relibra_attention_fwd(q1, k1, v, start, seq_len=length, err_flag=flag)
    o = out.flatten(1) @ D["Wo"].T
    x_out, n_out = rl.relibra_block_norm_fwd(D["x"], y=o, w_post=D["w2"], w_pre=D["w3"], gate=D["g"], res_scale=RHO, eps=EPS)

    # ---- backward, the projection's gradient in one tensor
    dx, do, dg, dw2, dw3 = rl.relibra_block_norm_bwd(x_out, up_x.to(DEV), up_n.to(DEV), y=o, w_post=D["w2"], w_pre=D["w3"], gate=D["g"], res_scale=RHO, eps=EPS)
    dout = (do @ D["Wo"]).unflatten(1, (Hq, d))
    dWo = do.float().T @ out.flatten(1).float()
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = parts(dqkv)
    rl.relibra_attention_bwd(q1, k1, v, out, lse, dout, start, seq_len=length, dq=dq, dk=dk, dv=dv, err_flag=flag)
    _, _, dwq, dwk = rl.relibra_qk_norm_rope_bwd(q, k, dq, dk, **turn, dq=dq, dk=dk)      # in place
    dWqkv = dqkv.float().T @ n.float()
    dn = dqkv @ D["Wqkv"]
    dx, _, _, _, dw1 = rl.relibra_block_norm_bwd(D["x"], dx, dn, w_pre=D["w1"], eps=EPS)
    torch.cuda.synchronize()
    assert flag.item() == 0

    # ---- the same in double
    ref = {name: t.double().requires_grad_(True) for name, t in p.items()}
    angle = (pos.double()[torch.tensor(axis if axis else [0] * (rot // 2))].T * freq.double())
    want_x, want_n, goal = reference(ref, angle, list(zip(starts, lens)), Hq, Hk, d, up_x.double(), up_n.double())
    goal.backward()
    live = real.bool()
    rel = lambda a, w: float((a.cpu().double() - w.detach()).norm() / w.detach().norm())
    errs = dict(x_out=rel(x_out[live.to(DEV)], want_x[live]), n_out=rel(n_out[live.to(DEV)], want_n[live]), dx=rel(dx, ref["x"].grad), dw1=rel(dw1, ref["w1"].grad), dw2=rel(dw2, ref["w2"].grad),
                dw3=rel(dw3, ref["w3"].grad), dg=rel(dg, ref["g"].grad), dWo=rel(dWo, ref["Wo"].grad), dWqkv=rel(dWqkv, ref["Wqkv"].grad), dwq=rel(dwq, ref["wq"].grad), dwk=rel(dwk, ref["wk"].grad))
    assert max(errs.values()) <= TOL, errs
    assert torch.all(dqkv[~live.to(DEV)] == 0)                # padding has no gradient
