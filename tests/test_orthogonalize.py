"""Orthogonalised updates against the same steps in double precision.

Tolerance.  Operands are rounded to halves, 2^-11 of their value at most and 2e-4 in the root mean square.  In one step that
rounding enters A through both operands, B through A and A^2, and the product B X through both of its own; with singular values
around 1 the step magnifies these by about 5 sqrt(2), 5, 2.8 and 2.8 (|b| + 2 |c| |A| less what cancels; |B| <= 2.81): together
2e-4 * sqrt(50 + 25 + 8 + 8) = 1.9e-3 of the result's norm.  The steps behind it pass an error on with |p'| about 1 (0.7 at 1,
1.1 at 0.7), so five steps leave sqrt(5) * 1.9e-3 = 4.3e-3, and rounding the result to bf16 adds 1.7e-3: TOL = 6e-3 of the norm.  The
linear term has 22 bits, so what lies outside of a low-rank gradient's space, magnified 485 times, stays below 485 * 2^-22 =
1.2e-4.  Single values: six of these root mean squares, where no value stands out."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
TOL = 6e-3
A, B, K = 3.4445, -4.7750, 2.0315


def definition(u, steps=5, scale=1.0):
    """u [n, r, c] double -> the update, matrix by matrix."""
    out = []
    for x in u.double():
        norm = x.norm()
        x = x / norm if norm > 0 else x
        for _ in range(steps):
            g = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
            p = B * g + K * (g @ g)
            x = A * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
        out.append(scale * x)
    return torch.stack(out)


def gauss(n, r, c, seed=0):
    return torch.randn((n, r, c), generator=torch.Generator().manual_seed(seed))


def close(got, want, tol=TOL):
    got, want = got.cpu().double(), want.double()
    assert torch.isfinite(got).all()
    for g, w in zip(got, want):
        n = w.norm()
        assert (g - w).norm() <= tol * n, float((g - w).norm() / n)


SHAPES = [(1, 1, 1), (3, 1, 7), (2, 9, 1), (2, 64, 64), (1, 63, 65), (4, 128, 256), (3, 256, 128), (2, 257, 130), (1, 300, 1000), (1, 1001, 333), (2, 512, 520), (1, 640, 576),
          (9, 320, 257), (1, 40, 4100), (1, 4100, 24), (70, 33, 47), (1, 1100, 1030),
          (3, 128, 1000), (2, 700, 127), (40, 128, 520), (200, 300, 64), (1, 65, 9000), (600, 16, 40), (5, 129, 128), (2, 128, 128),
          (1, 200, 2500), (3, 2049, 150), (1, 260, 5000), (2, 8200, 140)]


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_orthogonalize_against_double_precision(shape, dtype):
    g = (1e-3 * gauss(*shape, seed=sum(shape))).to(dtype)
    out, mom = rl.relibra_orthogonalize(g.to(DEV), scale=0.2 * math.sqrt(max(shape[1:])))
    assert mom is None and out.dtype == torch.bfloat16
    close(out, definition(g, scale=0.2 * math.sqrt(max(shape[1:]))))


def spectrum(r, c, s, seed):
    g = torch.Generator().manual_seed(seed)
    m = min(r, c)
    u = torch.linalg.qr(torch.randn((r, m), generator=g, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn((c, m), generator=g, dtype=torch.float64))[0]
    return (u * s) @ v.T


@gpu
@pytest.mark.parametrize("shape", [(192, 448), (448, 192), (384, 384)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", ["rank1", "rank4", "decay", "steep", "one_large"])
def test_orthogonalize_gradients_of_few_dimensions(shape, kind):
    m = min(shape)
    s = torch.zeros(m, dtype=torch.float64)
    if kind == "rank1":
        s[0] = 1
    elif kind == "rank4":
        s[:4] = torch.tensor([1.0, 0.5, 0.3, 0.2])
    elif kind == "decay":
        s = torch.logspace(0, -6, m, dtype=torch.float64)
    elif kind == "steep":
        s[:40] = torch.logspace(0, -3, 40, dtype=torch.float64)
    else:
        s[:] = 1e-3
        s[0] = 1
    g = spectrum(*shape, s, 5)[None].float()
    out, _ = rl.relibra_orthogonalize(g.to(DEV))
    close(out, definition(g))
    # and what it is for: the leading singular values end up near 1
    top = torch.linalg.svdvals(out[0].cpu().double())[: max(1, int((s > 0.05 * s.norm()).sum()))]
    assert torch.all((top > 0.6) & (top < 1.3)), top


@gpu
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 130, 200), (2, 65, 33)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_momentum(shape, dtype, nesterov):
    mu = 0.9
    mom = gauss(*shape, seed=1)
    mom_d = mom.to(DEV)
    for step in range(3):
        g = gauss(*shape, seed=2 + step).to(dtype)
        want_m = mu * mom_d.cpu().double() + g.double()
        u = g.double() + mu * want_m if nesterov else want_m
        out, got_m = rl.relibra_orthogonalize(g.to(DEV), momentum=mom_d, mu=mu, nesterov=nesterov, momentum_out=mom_d if step else None)
        # the fp32 value of 0.9 and one rounding of the sum
        assert torch.all((got_m.cpu().double() - want_m).abs() <= 2.0 ** -24 * (2 * want_m.abs() + 2 * mom_d.abs().max().item()))
        close(out, definition(u))
        mom_d = got_m


@gpu
def test_orthogonalize_zero_huge_tiny_and_nan_matrices_side_by_side():
    g = gauss(7, 100, 70, seed=3)
    g[1] = 0
    g[2] *= 1e30
    g[3] *= 1e-36
    g[4, 5, 6] = math.nan
    g[5, 0, 0] = math.inf
    out, _ = rl.relibra_orthogonalize(g.to(DEV))
    keep = [0, 2, 3, 6]
    close(out[keep], definition(g[keep]))
    assert torch.all(out[1] == 0) and torch.isnan(out[4].float()).any() and torch.isnan(out[5].float()).any()


@gpu
@pytest.mark.parametrize("steps", [1, 2, 8])
def test_orthogonalize_other_numbers_of_steps(steps):
    g = gauss(2, 96, 160, seed=4)
    close(rl.relibra_orthogonalize(g.to(DEV), steps=steps)[0], definition(g, steps))


@gpu
def test_orthogonalize_sizes_of_zero():
    for shape in ((0, 4, 4), (3, 0, 5), (3, 5, 0)):
        assert rl.relibra_orthogonalize(torch.zeros(shape, device=DEV))[0].shape == shape


@gpu
def test_orthogonalize_is_reproducible_in_graphs_and_on_other_streams():
    """One workspace used by an eager call, a graph and its replays in turn; a matrix's result does not depend on the others' number."""
    g = gauss(6, 300, 520, seed=6).to(DEV)
    mom = gauss(6, 300, 520, seed=7).to(DEV)
    ws = rl.orthogonalize_workspace(6, 300, 520)
    src, out, mo = g.clone(), torch.empty_like(g, dtype=torch.bfloat16), torch.empty_like(mom)
    call = lambda: rl.relibra_orthogonalize(src, momentum=mom, out=out, momentum_out=mo, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for turn in range(3):
        src.copy_(g * (turn + 1))
        want, want_m = rl.relibra_orthogonalize(src.clone(), momentum=mom)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(mo, want_m), turn
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again, _ = rl.relibra_orthogonalize(src[2:3].contiguous(), momentum=mom[2:3].contiguous())
        side.synchronize()
        close(again, definition((src[2:3].double() + 0.95 * want_m[2:3].double()).cpu()))


# ------------------------------------------------------------------ refusals (no GPU needed: nothing is launched)
def _call(grad=4096, mom=0, n=2, rows=64, cols=64, steps=5, flags=0, mom_out=0, out=8192, ws=4096, ws_bytes=1 << 40):
    p, f = C.c_void_p, C.c_float
    return rl.lib().relibra_orthogonalize(p(grad), p(mom), n, rows, cols, f(0.9), f(1), steps, flags, p(mom_out), p(out), p(ws), C.c_size_t(ws_bytes), p(0))


def test_orthogonalize_refusals():
    for bad in (dict(n=-1), dict(rows=-1), dict(cols=-1), dict(steps=0), dict(flags=4), dict(grad=0), dict(out=0), dict(out=4096), dict(ws=4104), dict(mom=4096),
                dict(mom_out=4096), dict(flags=2)):
        assert _call(**bad) == rl.EINVAL, bad
    for bad in (dict(n=65536), dict(rows=32769), dict(cols=32769), dict(steps=65)):
        assert _call(**bad) == rl.EUNSUPPORTED, bad
    need = rl.workspace_bytes(rl.WS_ORTHOGONALIZE, 0, 1, 2, 1, 64, 64)
    assert need > 0 and _call(ws_bytes=need - 1) == rl.EWORKSPACE and _call(ws=0) == rl.EWORKSPACE
    for none in (dict(n=0), dict(rows=0), dict(cols=0)):
        assert _call(**none) == rl.OK, none


@gpu
@pytest.mark.parametrize("shape", [(40, 300, 520), (40, 520, 300), (28, 400, 527), (28, 527, 400), (16, 600, 600)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_many_matrices(shape):
    """Enough tiles for each of the tile sizes, of which the last of a matrix is not whole."""
    g = 1e-3 * gauss(*shape, seed=sum(shape))
    out, mom = rl.relibra_orthogonalize(g.to(DEV), momentum=torch.zeros(shape, device=DEV), nesterov=False)
    assert torch.equal(mom.cpu(), g)
    close(out, definition(g))


@gpu
@pytest.mark.parametrize("shape", [(1, 32768, 136), (2, 140, 32768), (1, 32768, 24), (1, 1, 32768)], ids=lambda s: "x".join(map(str, s)))
def test_orthogonalize_longest_sides(shape):
    g = 1e-3 * gauss(*shape, seed=sum(shape))
    out, _ = rl.relibra_orthogonalize(g.to(DEV))
    close(out, definition(g))


def test_orthogonalize_no_workspace_for_unusable_sizes():
    for n, rows, cols in ((1, 32769, 8), (1, 8, 32769), (65536, 8, 8), (1, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert rl.workspace_bytes(rl.WS_ORTHOGONALIZE, 0, 1, n, 1, rows, cols) == 0
