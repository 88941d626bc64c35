"""Orthogonalised updates value by value, against the same steps in double precision and a simulation of the kernels' roundings.

Tolerance.  `rounded` takes the steps in double precision and rounds where the kernels round: X to two halves of which the first enters
products, A and B to halves with their diagonals left out, and sums to fp32.  A sum of m products that is rounded after every 8 of them is off by
2^-24 sqrt(m / 8) of its size or so, which is small beside the halves but not beside the second half of X (2^-22), and leaves a low-rank gradient's
space just so: without it the simulation has half of the noise that 8 steps magnify at m = 256 (8e-4 of the norm for 1.5e-3).  What `rounded` differs by
from `definition` is the error before the result's own rounding to bf16; the kernels add in another order, which moves values
across rounding borders now and then: LIKE = 1.5 times the simulated error is allowed.  Rounding to bf16 adds at most half a step to a value, 2^-8 of it; over a matrix the
squares of N independent half steps h_i add up to sum h_i^2 / 3 give or take SIGMAS = 6 standard deviations sqrt(4/45 sum h_i^4).  A single value is allowed
SIGMAS root mean squares of the simulated error besides its half step: it fails a value that is missing unless that value is nearly 0."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
SCALE = 4096.0
LIKE, SIGMAS = 1.5, 6.0
HALF16 = torch.finfo(torch.bfloat16).eps / 2


def gauss(n, r, c, seed=0):
    return torch.randn((n, r, c), generator=torch.Generator().manual_seed(seed))


def low_rank(n, r, c, rank, seed=0):
    return torch.bmm(gauss(n, r, rank, seed), gauss(n, rank, c, seed + 1))


def definition(u, steps):
    """One matrix in double precision, the longer side along the rows."""
    x = u.double() / u.double().norm()
    for _ in range(steps):
        a = x @ x.T
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    return x


def product(p, q):
    total = torch.zeros((p.shape[0], q.shape[1]), dtype=torch.float64)
    for k in range(0, p.shape[1], 8):
        total = (total + p[:, k:k + 8] @ q[k:k + 8]).float().double()
    return total


def rounded(u, steps, apart=True):
    """The same with the kernels' roundings; apart: the diagonals of A and B do not go through halves."""
    half = lambda t: t.half().double()
    split = lambda t: (half(t), half(t - half(t)))
    off = lambda t: t - torch.diag(torch.diag(t)) if apart else t
    dia = lambda t: torch.diag(t) if apart else torch.zeros(len(t), dtype=t.dtype)
    x = u.double() / u.double().norm() * SCALE
    hi, lo = split(x)
    for i in range(steps):
        a = product(hi, hi.T.contiguous()) / SCALE
        d, a = dia(a), half(off(a))
        p = product(a, a)
        b = NS_B * a + NS_C / SCALE * (p + (d[:, None] + d[None, :]) * a)
        db = (dia(b) + NS_B * d + NS_C / SCALE * d * d)[:, None] / SCALE
        weight = 1.0 if i + 3 >= steps else 0.0
        x = (NS_A + db) * hi + (NS_A + weight * db) * lo + product(half(off(b)), hi) / SCALE
        hi, lo = split(x)
    return x / SCALE


def wide(u):
    return u.T if u.shape[0] > u.shape[1] else u


def check_values(got, u, steps=5, scale=1.0, single=True):
    """got [n, r, c] bf16 of the matrices u.  single: value by value too (where the error is spread evenly: not for few dimensions)."""
    assert got.shape == u.shape and got.dtype == torch.bfloat16
    for i, (g, m) in enumerate(zip(got.cpu().double(), u)):
        want = scale * definition(wide(m), steps)
        error = (scale * rounded(wide(m), steps) - want).norm()
        off = wide(g) - want
        assert torch.isfinite(g).all(), i
        h2 = torch.exp2(2 * torch.floor(torch.log2(want.abs().clamp(min=1e-38)))) * HALF16 ** 2
        allowed = h2.sum() / 3 + SIGMAS * torch.sqrt(4 / 45 * (h2 * h2).sum()) + (LIKE * error) ** 2
        assert off.norm() ** 2 <= allowed, (i, float(off.norm() / want.norm()), float(allowed.sqrt() / want.norm()))
        if single:
            limit = HALF16 * want.abs() + (1 + HALF16) * SIGMAS * LIKE * error / math.sqrt(want.numel())
            assert torch.all(off.abs() <= limit), (i, float((off.abs() / limit).max()), int((off.abs() > limit).sum()))


# ------------------------------------------------------------------ the check itself: mistakes in the oracle are seen
@pytest.mark.parametrize("shape", [(64, 1000), (128, 256), (333, 1001), (136, 2000)], ids=lambda s: "x".join(map(str, s)))
def test_the_check_sees_missing_lines_pieces_and_diagonals(shape):
    u = gauss(1, *shape, seed=3)
    good = rounded(u[0], 5)[None].to(torch.bfloat16)
    check_values(good, u)
    for cut in ((0, slice(None), -1), (0, -1, slice(None)), (0, 5, slice(8, 16)), (0, slice(8, 9), 7)):
        bad = good.clone()
        bad[cut] = 0
        with pytest.raises(AssertionError):
            check_values(bad, u)
    with pytest.raises(AssertionError):                      # diagonals through halves
        check_values(rounded(u[0], 5, apart=False)[None].to(torch.bfloat16), u)


# ------------------------------------------------------------------ numbers of steps
FEW = [(256, 500), (500, 256), (100, 300), (300, 100), (40, 2000), (128, 128)]      # tiles and thin, wide and tall


@gpu
@pytest.mark.parametrize("shape", FEW, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("rank", [1, 4, 16])
@pytest.mark.parametrize("steps", [5, 8])
def test_orthogonalize_few_dimensions_up_to_the_last_step(shape, rank, steps):
    """What rounding leaves outside of the gradient's space grows by 3.44 a step; up to 8 steps the result is the definition's
    (simulated: at most 3.2e-3 of the norm for these)."""
    u = low_rank(2, *shape, rank, seed=rank)
    out, _ = rl.relibra_orthogonalize(u.to(DEV), steps=steps)
    check_values(out, u, steps, single=False)
    for g, m in zip(out.cpu().double(), u):
        want = definition(wide(m), steps)
        assert (wide(g) - want).norm() <= 4e-3 * want.norm()


@gpu
@pytest.mark.parametrize("shape", FEW, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("steps", [1, 3, 8])
def test_orthogonalize_every_number_of_steps_has_its_own_end(shape, steps):
    u = gauss(3, *shape, seed=steps)
    check_values(rl.relibra_orthogonalize(u.to(DEV), steps=steps)[0], u, steps)


def call(n=2, rows=64, cols=64, steps=5, flags=0, grad=1 << 20, mom=0, mom_out=0, out=2 << 20, ws=4 << 20, ws_bytes=1 << 40):
    """A call that has to be refused: nothing is launched, no pointer is followed."""
    p, f = C.c_void_p, C.c_float
    return rl.lib().relibra_orthogonalize(p(grad), p(mom), n, rows, cols, f(0.9), f(1), steps, flags, p(mom_out), p(out), p(ws), C.c_size_t(ws_bytes), p(0))


@pytest.mark.parametrize("steps", [9, 12, 64])
def test_orthogonalize_refuses_steps_whose_result_would_be_noise(steps):
    """Rank 1 of 256 x 500, simulated: 1.6e-2 of the norm after 10 steps, 0.2 after 12."""
    assert call(steps=steps) == rl.EUNSUPPORTED


def test_no_workspace_for_sizes_that_the_calls_refuse():
    for n, rows, cols in ((65535, 32768, 32768), (4096, 32768, 32768), (65535, 32768, 2049)):
        assert call(n=n, rows=rows, cols=cols) == rl.EUNSUPPORTED
        assert rl.workspace_bytes(rl.WS_ORTHOGONALIZE, 0, 1, n, 1, rows, cols) == 0
    assert rl.workspace_bytes(rl.WS_ORTHOGONALIZE, 0, 1, 4095, 1, 32768, 32768) > 0
    assert rl.workspace_bytes(rl.WS_ROUTER, 4, 65, 128, 1, 0, 0) == 0 and rl.workspace_bytes(rl.WS_ROUTER, 4, 9, 8, 1, 0, 0) == 0
    assert rl.workspace_bytes(rl.WS_ROUTER, 4, 64, 128, 1, 0, 0) > 0 and rl.workspace_bytes(rl.WS_ROUTER, 4, 8, 8, 1, 0, 0) > 0


def test_orthogonalize_refuses_outputs_over_inputs():
    """2 matrices of 64 x 64: 32 KiB in fp32, 16 KiB in bf16.  A momentum written over the gradient would be read as the gradient."""
    grad, mom, out, k = 1 << 20, 8 << 20, 2 << 20, 1 << 10
    for flags in (0, rl.ORTHO_NESTEROV):
        with_momentum = dict(mom=mom, flags=flags)
        for at in (grad, grad + 4, grad + 32 * k - 4, grad - 32 * k + 4, mom + 4, mom - 4):
            assert call(mom_out=at, **with_momentum) == rl.EINVAL, at
        for at in (mom, mom + 32 * k - 2, mom - 16 * k + 2, grad + 2):
            assert call(mom_out=mom, out=at, **with_momentum) == rl.EINVAL, at
        assert call(mom_out=16 << 20, out=(16 << 20) + 8 * k, **with_momentum) == rl.EINVAL
        assert call(mom_out=grad + 8 * k, grad=grad, mom=mom, flags=flags | rl.ORTHO_BF16) == rl.EINVAL
    assert call(out=grad) == rl.EINVAL and call(out=grad - 16 * k + 2) == rl.EINVAL and call(out=grad + 16 * k - 2, flags=rl.ORTHO_BF16) == rl.EINVAL


# ------------------------------------------------------------------ every path, every value, nothing else
def guarded(shape, dtype, odd=0):
    """A tensor of NaN bits with 64 (+ odd) elements of them in front and 64 behind, and a check that those are as they were."""
    count = math.prod(shape)
    ints = {2: torch.int16, 4: torch.int32, 1: torch.uint8}[dtype.itemsize]
    flat = torch.full((count + 128 + odd,), 255 if dtype.itemsize == 1 else -1, dtype=ints, device=DEV)
    whole = flat.view(dtype)

    def untouched():
        edge = torch.cat([flat[:64 + odd], flat[64 + odd + count:]])
        return bool((edge == (255 if dtype.itemsize == 1 else -1)).all())
    return whole[64 + odd:64 + odd + count].view(shape), untouched


PATHS = [
    # a short side of at most 64 (runs of 256 rows): one workgroup a matrix; several runs each; several workgroups, their sums direct or summed first
    (3, 1, 7), (2, 9, 1), (1, 1, 300), (9, 33, 47), (300, 16, 40), (130, 50, 600), (200, 300, 64), (2, 64, 700), (1, 24, 4100), (40, 2000, 60), (100, 2500, 33),
    # at most 128 (runs of 128 rows): the same
    (4, 128, 256), (5, 65, 66), (130, 100, 300), (130, 300, 100), (2, 127, 700), (1, 1000, 128), (100, 127, 700), (100, 700, 127), (40, 127, 1500), (40, 1500, 127),
    # few tiles, wide and tall, contraction whole and split (2112: four parts; 4672: nine, the last of one LDS tile)
    (2, 257, 130), (1, 300, 1000), (3, 1001, 333), (1, 300, 2112), (1, 2112, 300), (1, 260, 4672), (1, 4672, 140), (5, 129, 192),
    # small tiles for X' where they are more: 216 of 128 x 128, 72 of 256 x 256
    (6, 300, 1500), (6, 1500, 300),
    # X' in large tiles, A and B in small ones of single depth (more than 256 of them) and in large ones
    (28, 400, 527), (28, 527, 400), (40, 300, 520), (44, 500, 310),
]


@gpu
@pytest.mark.parametrize("shape", PATHS, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("odd", [0, 1], ids=["aligned", "odd"])
def test_orthogonalize_writes_every_value_and_nothing_else(shape, odd):
    """Outputs and workspace full of NaN before the call, NaN around them; odd: outputs and inputs 2 or 4 bytes off 16."""
    n, r, c = shape
    dtype = torch.bfloat16 if odd else torch.float32
    g, m = gauss(*shape, seed=sum(shape)).to(dtype), gauss(*shape, seed=r)
    gd, md = guarded(shape, dtype, odd)[0].copy_(g), guarded(shape, torch.float32, odd)[0].copy_(m)
    out, out_kept = guarded(shape, torch.bfloat16, odd)
    mom, mom_kept = guarded(shape, torch.float32, odd)
    ws, ws_kept = guarded((rl.workspace_bytes(rl.WS_ORTHOGONALIZE, 0, 1, n, 1, r, c),), torch.uint8)
    rl.relibra_orthogonalize(gd, momentum=md, mu=0.5, nesterov=bool(odd), scale=0.3, out=out, momentum_out=mom, workspace=ws)
    torch.cuda.synchronize()
    assert out_kept() and mom_kept() and ws_kept()
    assert torch.equal(md.cpu(), m) and torch.equal(gd.cpu(), g)
    want_m = 0.5 * m.double() + g.double()
    assert torch.equal(mom.cpu(), want_m.float())            # (0.5 m is exact: one rounding)
    step = mom.cpu()
    u = torch.addcmul(g.double(), step.double(), torch.tensor(0.5, dtype=torch.float64)) if odd else step.double()
    some = [0, n // 2, n - 1] if n > 8 else range(n)
    check_values(out[list(some)], u[list(some)], scale=0.3)
    assert torch.isfinite(out.float()).all()


@gpu
@pytest.mark.parametrize("shape", [(3, 70, 40), (3, 100, 300), (3, 1, 50), (2, 300, 140), (2, 130, 700), (100, 127, 700)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_orthogonalize_infinities_and_nan_fill_their_own_matrix(shape, value):
    g = gauss(*shape, seed=9)
    g[1, shape[1] // 2, shape[2] - 1] = value
    out, _ = rl.relibra_orthogonalize(g.to(DEV))
    assert torch.isnan(out[1].float()).all() and torch.isfinite(out[0].float()).all() and torch.isfinite(out[2:].float()).all()
    check_values(out[:1], g[:1])


@gpu
@pytest.mark.parametrize("shape", [(1, 32768, 136), (2, 140, 16384), (1, 1, 32768), (1, 32768, 90), (1, 4096, 700)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_every_value_of_the_longest_sides(shape):
    g = 1e-3 * gauss(*shape, seed=sum(shape))
    check_values(rl.relibra_orthogonalize(g.to(DEV))[0], g)


@gpu
@pytest.mark.parametrize("shape", [(64, 1000), (1000, 64), (256, 256), (300, 700)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_values_of_one_size(shape):
    """Signs times signs: all values round alike, and their errors add up instead of averaging out."""
    g = (gauss(1, shape[0], 1, 1).sign() * gauss(1, 1, shape[1], 2).sign()).expand(2, *shape).contiguous()
    out, _ = rl.relibra_orthogonalize(g.to(DEV))
    for o in out.cpu().double():
        want = definition(wide(g[0]), 5)
        assert (wide(o) - want).norm() <= 1.3e-2 * want.norm()
