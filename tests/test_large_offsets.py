"""Tensors of more than 2^31 values through the operators of a training step: their last part against a call on that part alone.

A token's gates and gradient, and a row's norms and gradients, do not depend on the others, nor on how many blocks walk them: equal bit for
bit.  A matrix's squares are added up by another number of blocks where there are fewer matrices: a value may fall on the other side of
a rounding border in the first halves of X, 2^-11 of it at most, seldom; 1e-3 of the norm is allowed."""
import pytest
import torch

import paper_2605_08639_amd as rl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def noise(*shape, dtype=torch.bfloat16):
    """Standard normal values, made piece by piece in their own type."""
    return torch.empty(shape, dtype=dtype, device=DEV).normal_()


def test_router_of_many_tokens_and_experts():
    n_mb, T, E, k = 2, (1 << 18) + 77, 4096, 4
    assert n_mb * T * E > 1 << 31
    torch.manual_seed(1)
    z = noise(n_mb, T, E)
    ids = torch.randint(0, E, (n_mb, T, k), dtype=torch.int32, device=DEV)
    dg = torch.randn((n_mb, T, k), device=DEV)
    gates, counts, n_valid, mean, loss = rl.relibra_router_fwd(z, ids, balance_coef=1.0)
    dz = rl.relibra_router_bwd(z, ids, dg)
    last = (slice(1, 2), slice(T - 100, T))
    part = [t[last].contiguous() for t in (z, ids, dg)]
    assert torch.equal(rl.relibra_router_fwd(part[0], part[1])[0], gates[last])
    assert torch.equal(rl.relibra_router_bwd(*part), dz[last])
    assert torch.equal(counts.long(), torch.stack([torch.bincount(i.reshape(-1), minlength=E) for i in ids])) and n_valid.tolist() == [T, T]
    assert torch.isfinite(loss).all() and (mean.double().sum(1) - 1).abs().max().item() < 1e-5


def test_norms_of_many_rows():
    T, h = (1 << 18) + 333, 8192
    assert T * h > 1 << 31
    torch.manual_seed(2)
    x, y, gate = noise(T, h), noise(T, h), torch.rand(T, device=DEV)
    w2, w1 = noise(h), noise(h)
    x_out, n = rl.relibra_block_norm_fwd(x, y=y, w_post=w2, w_pre=w1, gate=gate)
    last = slice(T - 300, T)
    how = dict(y=y[last], w_post=w2, w_pre=w1, gate=gate[last].clone())
    a = rl.relibra_block_norm_fwd(x[last], **how)
    assert torch.equal(a[0], x_out[last]) and torch.equal(a[1], n[last])
    dx, dy, dgate, dw2, dw1 = rl.relibra_block_norm_bwd(x_out, x, n, y=y, w_post=w2, w_pre=w1, gate=gate)
    b = rl.relibra_block_norm_bwd(x_out[last], x[last], n[last], **how)
    assert torch.equal(b[0], dx[last]) and torch.equal(b[1], dy[last]) and torch.equal(b[2], dgate[last])
    assert torch.isfinite(dw1).all() and torch.isfinite(dw2).all()


@pytest.mark.parametrize("shape", [(520, 2048, 2048), (2100, 128, 8192)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalised_updates_of_many_values(shape):
    n = shape[0]
    assert shape[0] * shape[1] * shape[2] > 1 << 31
    torch.manual_seed(3)
    g = noise(*shape)
    mom = noise(*shape, dtype=torch.float32)
    out, new = rl.relibra_orthogonalize(g, momentum=mom, nesterov=False)
    last = slice(n - 260, n)
    part, part_new = rl.relibra_orthogonalize(g[last], momentum=mom[last], nesterov=False)
    assert torch.equal(part_new, new[last])
    for a, b in zip(part[-3:].double(), out[-3:].double()):
        assert b.norm().item() > 1 and ((a - b).norm() <= 1e-3 * b.norm()).item()


def test_orthogonalised_update_of_the_largest_matrix():
    """A Hadamard matrix: rows at right angles, values of one size, every singular value the same, so that the steps are those of a number.
    Values that all round alike: 1.3e-2 of the norm."""
    m = 32768
    i = torch.arange(m, device=DEV)
    sign = torch.ones((m, m), dtype=torch.bfloat16, device=DEV)
    for bit in range(15):                                    # (-1)^(number of ones in i and j)
        odd = ((i >> bit) & 1).bool()
        sign[odd] *= torch.where(odd, -1.0, 1.0).to(torch.bfloat16)
    s = m ** -0.5
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    out, _ = rl.relibra_orthogonalize(sign[None], scale=float(m ** 0.5))
    off = (out[0] * sign).float() - s
    assert off.abs().max().item() <= 1.3e-2 * s + 2.0 ** -8 * s
