"""Causal attention of packed sequences with grouped heads, and its gradients, against plain double precision.

Tolerances, for each value from the sizes of its terms (U = 2^-24 for fp32, H = 2^-8 for a rounding to bf16):
 * a score is a sum of d products: off by EZ = (d + 4) U scale sum |q||k|, its exponential by that of itself, twice (its own, the reference's) and 8 U more;
 * lse: EZ of the row, n U for the sum of n exponentials, 8 U |lse|;
 * out: every p is rounded to bf16 before its product with v (H), p's own error, n + 16 additions, the division, and one rounding of the result:
   (H + EP + (n + 24) U) sum p |v| + H |out|, with EP = 2 EZ + (n + 16) U the relative error of p;
 * D = do . out carries out's error: ED = sum |do| err(out);  dp: (d + 4) U sum |do||v|;  ds = p (dp - D): p (ED + err(dp)) + (EP + H) |ds| with EP from lse's error,
   and H more of p |dp - D| rounded to bf16;
 * dq, dk, dv: those times the other operand's sizes, summed, n + 16 additions, and one rounding."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_08639_amd as rl

DEV = "cuda"
gpu = pytest.mark.gpu
BF16 = torch.bfloat16
U = torch.finfo(torch.float32).eps / 2
H = torch.finfo(BF16).eps / 2


def make(places, Hk, G, d, lens=None, before=0, behind=0, seed=0, peak=1.5):
    """Sequences of `places` rows, the first lens of them tokens; rows before the first and behind the last belong to none."""
    g = torch.Generator().manual_seed(seed)
    T = before + sum(places) + behind
    r = lambda heads, size=1.0: (size * torch.randn(T, heads, d, generator=g)).to(BF16)
    starts = [before]
    for n in places:
        starts.append(starts[-1] + n)
    return dict(q=r(Hk * G, peak), k=r(Hk), v=r(Hk), dout=r(Hk * G), starts=starts, lens=list(places) if lens is None else lens, padded=lens is not None, scale=d ** -0.5,
                Hk=Hk, G=G, d=d, T=T)


def tables(c):
    return torch.tensor(c["starts"], dtype=torch.int32, device=DEV), torch.tensor(c["lens"], dtype=torch.int32, device=DEV) if c["padded"] else None


def run(c, bwd=True, **kw):
    """(out, lse, dq, dk, dv) of the library."""
    start, length = tables(c)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    flag = rl.new_err_flag()
    out, lse = rl.relibra_attention_fwd(d["q"], d["k"], d["v"], start, seq_len=length, scale=c["scale"], err_flag=flag, **kw)
    grads = rl.relibra_attention_bwd(d["q"], d["k"], d["v"], out, lse, d["dout"], start, seq_len=length, scale=c["scale"], err_flag=flag) if bwd else ()
    assert flag.item() == 0
    return (out, lse, *grads)


def check(c, got, bwd=True):
    out, lse = got[0].cpu().double(), got[1].cpu().double()
    covered = torch.zeros(c["T"], dtype=torch.bool)
    G, d, s = c["G"], c["d"], c["scale"]
    for start, end, n in zip(c["starts"], c["starts"][1:], c["lens"]):
        rows, pad = slice(start, start + n), slice(start + n, end)
        covered[rows] = True
        assert torch.all(out[pad] == 0) and torch.all(lse[pad] == 0)
        if bwd:
            assert all(torch.all(x.cpu()[pad] == 0) for x in got[2:])
        if n == 0:
            continue
        mask = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(c["Hk"]):
            k, v = c["k"][rows, h].double(), c["v"][rows, h].double()
            sums = [torch.zeros(n, d, dtype=torch.float64) for _ in range(4)]              # dk, dv and the sizes of their errors
            for g in range(h * G, (h + 1) * G):
                q, do = c["q"][rows, g].double(), c["dout"][rows, g].double()
                z = (s * q @ k.T).masked_fill(~mask, -math.inf)
                ez = ((d + 4) * U * s * (q.abs() @ k.abs().T)).masked_fill(~mask, 0).amax(1, keepdim=True)
                want_lse = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - want_lse)
                ep = 2 * ez + (n + 16) * U
                off = (lse[rows, g, None] - want_lse).abs()
                err_lse = ez + (n + 16) * U + 8 * U * want_lse.abs()
                assert torch.all(off <= err_lse), ("lse", float((off / err_lse).max()))
                want, size = p @ v, p @ v.abs()
                err_out = (H + ep + (n + 24) * U) * size + H * want.abs()
                off = (out[rows, g] - want).abs()
                assert torch.all(off <= err_out + 1e-30), ("out", g, float((off / err_out).max()))
                if not bwd:
                    continue
                dp, D = do @ v.T, (do * want).sum(1, keepdim=True)
                ds = (p * (dp - D)).masked_fill(~mask, 0)
                ep = ez + err_lse + 16 * U                    # p from the saved lse
                err_p = (H + ep) * p
                err_ds = (p * ((do.abs() * err_out).sum(1, keepdim=True) + (d + 8) * U * (do.abs() @ v.abs().T + (do.abs() * size).sum(1, keepdim=True))) + (2 * ep + H) * ds.abs()).masked_fill(~mask, 0)
                want_q = s * ds @ k
                err_q = s * (err_ds + (n + 24) * U * ds.abs()) @ k.abs() + H * want_q.abs()
                off = (got[2][rows, g].cpu().double() - want_q).abs()
                assert torch.all(off <= 1.01 * err_q + 1e-30), ("dq", g, float((off / err_q).max()))
                sums[0] += s * ds.T @ q
                sums[1] += p.T @ do
                sums[2] += s * (err_ds + (n * G + 24) * U * ds.abs()).T @ q.abs()
                sums[3] += (err_p + (n * G + 24) * U * p).T @ do.abs()
            if bwd:
                for name, x, want, err in (("dk", got[3], sums[0], sums[2]), ("dv", got[4], sums[1], sums[3])):
                    off, tol = (x[rows, h].cpu().double() - want).abs(), 1.01 * (err + H * want.abs()) + 1e-30
                    assert torch.all(off <= tol), (name, h, float((off / tol).max()))


CASES = dict(
    one_token=dict(places=[1], Hk=1, G=1, d=128), tokens=dict(places=[1, 1, 1, 2], Hk=2, G=2, d=64), tile_ends=dict(places=[63, 64, 65, 127, 128, 129], Hk=1, G=1, d=128),
    grouped_ends=dict(places=[7, 8, 9, 31, 32, 33], Hk=2, G=8, d=128), threes=dict(places=[200, 41, 1], Hk=2, G=3, d=80), fives=dict(places=[77, 130], Hk=1, G=5, d=72),
    wide_group=dict(places=[3, 70], Hk=1, G=64, d=64), small_heads=dict(places=[100, 300], Hk=3, G=1, d=8), d40=dict(places=[66, 190], Hk=2, G=2, d=40), d96=dict(places=[257], Hk=2, G=4, d=96),
    d104=dict(places=[129, 5], Hk=1, G=7, d=104), d32=dict(places=[513], Hk=4, G=1, d=32),
    empty_ones=dict(places=[0, 17, 0, 150, 0], Hk=2, G=2, d=64), padded=dict(places=[40, 130, 9, 300], lens=[33, 1, 0, 299], Hk=2, G=4, d=128, before=3, behind=6),
    padded_odd=dict(places=[200, 260], lens=[130, 129], Hk=1, G=3, d=88, before=1, behind=200), long=dict(places=[1400], Hk=1, G=2, d=128),
    shared_rows=dict(places=[700, 600], Hk=1, G=16, d=64), shared_rows_wide=dict(places=[640], Hk=1, G=24, d=120))


@gpu
@pytest.mark.parametrize("name", CASES)
def test_attention_against_the_definition(name):
    c = make(**CASES[name])
    check(c, run(c))


@gpu
@pytest.mark.parametrize("kw", [dict(Hk=2, G=3, d=72), dict(Hk=1, G=8, d=128), dict(Hk=2, G=1, d=32)], ids=str)
def test_attention_gradients_of_few_keys(kw):
    """Rows of a sequence's first 128 tokens: ds has twice bf16's bits (H^2 of it), and out's rounding is not in D.  D0, from the rounded out, is off by at most ED; D0 plus the sum
    of p (dp - D0) is D, but for p's relative error EP, the error of dp, and n + 16 additions: (EP + (n + 20) U) sum p |dp - D0| + sum p err(dp)."""
    c = make([1, 2, 3, 17, 64, 65, 100, 128], seed=31, **kw)
    out, lse, dq, dk, dv = (x.cpu().double() for x in run(c))
    G, d, s = c["G"], c["d"], c["scale"]
    for start, end in zip(c["starts"], c["starts"][1:]):
        rows, n = slice(start, end), end - start
        mask = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(c["Hk"]):
            k, v = c["k"][rows, h].double(), c["v"][rows, h].double()
            want_k, err_k = torch.zeros(n, d, dtype=torch.float64), torch.zeros(n, d, dtype=torch.float64)
            for g in range(h * G, (h + 1) * G):
                q, do = c["q"][rows, g].double(), c["dout"][rows, g].double()
                z = (s * q @ k.T).masked_fill(~mask, -math.inf)
                ez = ((d + 4) * U * s * (q.abs() @ k.abs().T)).masked_fill(~mask, 0).amax(1, keepdim=True)
                top = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - top)
                ep = ez + (ez + (n + 16) * U + 8 * U * top.abs()) + 16 * U
                want, size = p @ v, p @ v.abs()
                ED = (do.abs() * ((H + 2 * ez + (2 * n + 40) * U) * size + H * want.abs())).sum(1, keepdim=True)
                dp, D = do @ v.T, (do * want).sum(1, keepdim=True)
                err_dp = (d + 8) * U * (do.abs() @ v.abs().T + (do.abs() * size).sum(1, keepdim=True))
                err_D = (p * ((ep + (n + 20) * U) * ((dp - D).abs() + ED) + err_dp)).sum(1, keepdim=True)
                ds = (p * (dp - D)).masked_fill(~mask, 0)
                ds[0] = 0                                     # one key
                err_ds = p * (err_D + err_dp) + (2 * ep + H * H) * ds.abs()
                want_q = s * ds @ k
                err_q = s * (err_ds + (n + 24) * U * ds.abs()) @ k.abs() + H * want_q.abs()
                assert torch.all((dq[rows, g] - want_q).abs() <= 1.01 * err_q + 1e-30), ("dq", n, g)
                want_k += s * ds.T @ q
                err_k += s * (err_ds + (n * G + 24) * U * ds.abs()).T @ q.abs()
            assert torch.all((dk[rows, h] - want_k).abs() <= 1.01 * (err_k + H * want_k.abs()) + 1e-30), ("dk", n, h)


# Long sequences of few heads: tiles that several blocks share, in both directions; many heads of short ones: lists without shared tiles.
LONG = dict(
    two_heads=dict(places=[2100, 300], Hk=1, G=2, d=128), threes_padded=dict(places=[1300, 1400], lens=[1250, 1399], Hk=2, G=3, d=80, before=5, behind=9),
    eight_heads=dict(places=[3000], Hk=1, G=8, d=40), keys_of_their_own=dict(places=[64, 2300, 1], Hk=3, G=1, d=104), many_heads=dict(places=[300, 130, 270], lens=[300, 129, 260], Hk=512, G=1, d=8))


@gpu
@pytest.mark.parametrize("name", LONG)
def test_attention_of_long_sequences_and_many_heads(name):
    c = make(**LONG[name], seed=21)
    check(c, run(c))


def launches(c, **kw):
    """What run(c) gives, and how often each of the call's kernels was launched: (forward, backward)."""
    start, length = tables(c)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    count = []
    rl.prof_start(2)
    out, lse = rl.relibra_attention_fwd(d["q"], d["k"], d["v"], start, seq_len=length, scale=c["scale"])
    count.append({n: v[1] for n, v in rl.prof_stop().items() if v[1]})
    rl.prof_start(2)
    grads = rl.relibra_attention_bwd(d["q"], d["k"], d["v"], out, lse, d["dout"], start, seq_len=length, scale=c["scale"])
    count.append({n: v[1] for n, v in rl.prof_stop().items() if v[1]})
    return (out, lse, *grads), count


# A call of few sequences makes a list of its rows only where several blocks share their tiles; the keys' list is made beside the queries' kernel then.
SHARED = dict(
    d32=(dict(places=[2300, 100], Hk=1, G=2, d=32), True, True), d24_padded=(dict(places=[2500], lens=[2433], Hk=2, G=1, d=24), True, True),
    d8=(dict(places=[2400, 1], Hk=1, G=3, d=8), True, True), nine_heads=(dict(places=[1500, 1500, 1544], Hk=1, G=9, d=64), True, True),
    ten_heads=(dict(places=[1700, 2000, 396], lens=[1690, 2000, 390], Hk=1, G=10, d=32), True, True), twelve_heads=(dict(places=[1700, 1692], Hk=1, G=12, d=96), False, True),
    sixteen_heads=(dict(places=[1300, 1260], Hk=1, G=16, d=128), False, False))


@gpu
@pytest.mark.parametrize("name", SHARED)
def test_attention_of_tiles_that_blocks_share(name):
    kw, forward, backward = SHARED[name]
    c = make(**kw, seed=22)
    got, (fwd, bwd) = launches(c)
    assert [fwd.get("attn_sched", 0), fwd.get("attn_join", 0), bwd.get("attn_sched", 0), bwd.get("attn_join", 0)] == [forward, forward, backward, 1]
    check(c, got)


# The gradients' loads of rows move by a constant where a group divides what a load takes, 16 rows of heads above 64, 32 of others: on both sides of it and
# at it, with waves that begin inside of a group, last steps that are not whole, and padding.
GROUPS = dict(
    g16=dict(places=[1, 4, 5, 64, 130], Hk=1, G=16, d=128), g16_padded=dict(places=[90, 77], lens=[81, 3], Hk=2, G=16, d=128, before=4, behind=2), g16_d72=dict(places=[33, 70], Hk=2, G=16, d=72),
    g8_d104=dict(places=[9, 130], Hk=2, G=8, d=104), g32=dict(places=[1, 2, 3, 40, 65], Hk=1, G=32, d=64), g32_padded=dict(places=[50, 31], lens=[47, 30], Hk=2, G=32, d=40),
    g32_d128=dict(places=[7, 66], Hk=1, G=32, d=128), g24=dict(places=[20, 67], Hk=1, G=24, d=64), g64_d128=dict(places=[2, 35], Hk=1, G=64, d=128))


@gpu
@pytest.mark.parametrize("name", GROUPS)
def test_attention_of_wide_groups(name):
    c = make(**GROUPS[name], seed=23)
    check(c, run(c))


@gpu
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("n_seq,most", [(17, 9), (17, 90), (63, 4), (64, 5), (64, 40), (65, 5), (65, 40)])
def test_attention_on_both_sides_of_the_sequences_that_need_no_list(n_seq, most, G):
    """Blocks find their rows and keys in the tables for up to 64 sequences, one a lane; the keys' list of as many is made beside the queries' kernel where they are not few.  With padding and empty
    sequences among them, the last one too."""
    g = torch.Generator().manual_seed(n_seq + most)
    places = [int(x) for x in torch.randint(0, most + 1, (n_seq,), generator=g)]
    places[n_seq // 2], places[-2:] = 0, [most, 0 if G == 1 else most]
    lens = [int(torch.randint(0, p + 1, (1,), generator=g)) for p in places]
    lens[-2] = most
    c = make(places, 2, G, 64, lens=lens, before=1, behind=3, seed=24)
    got, (fwd, bwd) = launches(c)
    few = c["T"] * G <= 512
    assert [fwd.get("attn_sched", 0), bwd.get("attn_sched", 0), bwd.get("attn_join", 0)] == [n_seq > 64, n_seq > 64, n_seq > 64 or not few]
    check(c, got)

@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", ["peaked", "rising", "falling", "flat", "huge"])
def test_attention_scores_of_every_shape(shape, d):
    """Maxima that keep rising along the keys, that come first, one key that takes all, equal scores, scores of hundreds below zero."""
    c = make([300, 65], 1, 2, d, seed=3, peak=12.0 if shape == "peaked" else 1.0)
    if shape in ("rising", "falling"):
        for a, b in zip(c["starts"], c["starts"][1:]):
            ramp = torch.linspace(-1, 1, b - a) * (8 if shape == "rising" else -8)
            c["k"][a:b] = (ramp[:, None, None] + 0.1 * c["k"][a:b].float()).to(BF16)
        c["q"] = c["q"].abs()
    if shape == "flat":
        c["q"].zero_()
    if shape == "huge":
        c["q"] = (c["q"].abs() * 8).to(BF16)
        c["k"] = -c["k"].abs()
    check(c, run(c))


@gpu
def test_attention_of_a_fused_projection_and_into_one():
    """Parts of one tensor in, gradients into parts of one tensor: the same bits, nothing beside them written."""
    c = make([90, 130], 2, 4, 128, lens=[90, 77], seed=4)
    want = run(c)
    T, d, heads = c["T"], c["d"], (8, 2, 2)

    def fused(extra=8):
        whole = torch.full((T, sum(heads) * d + extra), 7.0, dtype=BF16, device=DEV)
        at, parts = 0, []
        for h in heads:
            parts.append(whole[:, at:at + h * d].unflatten(1, (h, d)))
            at += h * d
        return whole, parts
    _, parts = fused()
    for p, n in zip(parts, ("q", "k", "v")):
        p.copy_(c[n])
    start, length = tables(c)
    out, lse = rl.relibra_attention_fwd(*parts, start, seq_len=length)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    dwhole, dparts = fused()
    owide = torch.full((T, 10 * d), 7.0, dtype=BF16, device=DEV)
    o = owide[:, d:9 * d].unflatten(1, (8, d))
    rl.relibra_attention_fwd(*parts, start, seq_len=length, out=o)
    assert torch.equal(o, want[0]) and torch.all(owide[:, :d] == 7) and torch.all(owide[:, 9 * d:] == 7)
    got = rl.relibra_attention_bwd(*parts, o, lse, c["dout"].to(DEV), start, seq_len=length, dq=dparts[0], dk=dparts[1], dv=dparts[2])
    assert got[0] is dparts[0] and all(torch.equal(a, b) for a, b in zip(got, want[2:])) and torch.all(dwhole[:, sum(heads) * d:] == 7)


@gpu
def test_attention_first_tokens_have_no_gradient_of_scores():
    c = make([1, 5, 1], 1, 2, 64, seed=5)
    _, _, dq, dk, dv = run(c)
    for t in (0, 1, 6):
        assert torch.all(dq[t] == 0)
    for t in (0, 6):
        assert torch.all(dk[t] == 0)
        both = c["dout"][t].double().sum(0)                   # p is 1: dv is the sum over the group, one rounding
        assert torch.all((dv[t, 0].cpu().double() - both).abs() <= H * both.abs() + 4 * U * c["dout"][t].double().abs().sum(0))


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_attention_keeps_nan_and_infinities_where_they_are_seen(bad):
    """In padding, outside of all sequences: nobody notices.  In a token: its own sequence only, and no row more than 127 tokens before it."""
    kw = dict(places=[100, 400, 70], lens=[90, 390, 70], Hk=1, G=2, d=64, before=5, behind=9, seed=6)
    c = make(**kw)
    want = run(c)
    seen = torch.zeros(c["T"], dtype=torch.bool)
    for a, n in zip(c["starts"], c["lens"]):
        seen[a:a + n] = True
    for n in ("q", "k", "v", "dout"):
        c[n][~seen] = bad
    got = run(c)
    inside = slice(5, 575)
    assert all(torch.equal(a[inside], b[inside]) for a, b in zip(got, want))
    c = make(**kw)
    hit = c["starts"][1] + 300
    for n in ("k", "v"):
        c[n][hit] = bad
    got = run(c)
    assert torch.isnan(got[0][hit:c["starts"][1] + 390].float()).any(2).any(1).all() if bad != bad else not torch.isfinite(got[0][hit].float()).all()
    other = [slice(5, hit - 127), slice(c["starts"][2], 575)]
    assert all(torch.equal(a[part], b[part]) for a, b in zip(got[:2], want[:2]) for part in other)
    assert all(torch.equal(a[other[1]], b[other[1]]) for a, b in zip(got[2:], want[2:]))
    assert all(torch.equal(a[5:c["starts"][1]], b[5:c["starts"][1]]) for a, b in zip(got[2:], want[2:]))


@gpu
def test_attention_writes_every_value_and_nothing_else():
    c = make([64, 33, 200], 2, 3, 72, lens=[64, 20, 150], before=2, behind=4, seed=7)
    want = run(c)
    start, length = tables(c)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    n_seq, Hq = 3, 6
    outs = []
    for w in want:
        flat = torch.full((w.numel() + 128,), float("nan"), dtype=w.dtype, device=DEV)
        outs.append((flat, flat[64:-64].view(w.shape)))
    def space(which):
        ws = torch.full((rl.workspace_bytes(which, c["T"], 1, Hq, n_seq, 2, 72) + 256,), 255, dtype=torch.uint8, device=DEV)
        return ws, ws[:-256]
    (fw, f), (bw, b) = space(rl.WS_ATTENTION_FWD), space(rl.WS_ATTENTION_BWD)
    rl.relibra_attention_fwd(d["q"], d["k"], d["v"], start, seq_len=length, out=outs[0][1], lse=outs[1][1], workspace=f)
    rl.relibra_attention_bwd(d["q"], d["k"], d["v"], outs[0][1], outs[1][1], d["dout"], start, seq_len=length, dq=outs[2][1], dk=outs[3][1], dv=outs[4][1], workspace=b)
    inside = slice(2, c["T"] - 4)
    for (flat, got), w in zip(outs, want):
        assert torch.equal(got[inside], w[inside]) and torch.isnan(got[:2].float()).all() and torch.isnan(got[-4:].float()).all()
        assert torch.isnan(flat[:64].float()).all() and torch.isnan(flat[-64:].float()).all()
    assert torch.all(fw[-256:] == 255) and torch.all(bw[-256:] == 255)


@gpu
@pytest.mark.parametrize("start,length", [([0, 30, 20, 60], None), ([-1, 30, 40, 60], None), ([0, 30, 40, 61], None), ([0, 30, 40, 60], [30, 11, 20]), ([0, 30, 40, 60], [30, -1, 20]),
                                          ([0, 1 << 30, -(1 << 31), 60], None)])
def test_attention_flags_bad_tables_and_computes_nothing(start, length):
    c = make([30, 10, 20], 1, 2, 64, seed=8)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    start = torch.tensor(start, dtype=torch.int32, device=DEV)
    length = None if length is None else torch.tensor(length, dtype=torch.int32, device=DEV)
    out, lse = torch.full((60, 2, 64), 3.0, dtype=BF16, device=DEV), torch.full((60, 2), 3.0, device=DEV)
    flag = rl.new_err_flag()
    rl.relibra_attention_fwd(d["q"], d["k"], d["v"], start, seq_len=length, out=out, lse=lse, err_flag=flag)
    assert flag.item() == rl.ERR_SEQ_TABLE and torch.all(out == 3) and torch.all(lse == 3)
    flag.zero_()
    grads = [torch.full((60, h, 64), 3.0, dtype=BF16, device=DEV) for h in (2, 1, 1)]
    rl.relibra_attention_bwd(d["q"], d["k"], d["v"], out, lse, d["dout"], start, seq_len=length, dq=grads[0], dk=grads[1], dv=grads[2], err_flag=flag)
    assert flag.item() == rl.ERR_SEQ_TABLE and all(torch.all(g == 3) for g in grads)


@gpu
def test_attention_of_nothing():
    e = lambda h: torch.empty((0, h, 64), dtype=BF16, device=DEV)
    zero = torch.zeros(3, dtype=torch.int32, device=DEV)
    out, lse = rl.relibra_attention_fwd(e(2), e(1), e(1), zero)
    assert out.shape == (0, 2, 64) and rl.relibra_attention_bwd(e(2), e(1), e(1), out, lse, e(2), zero)[1].shape == (0, 1, 64)
    c = make([5], 1, 2, 64)
    q, k, v = (c[n].to(DEV) for n in ("q", "k", "v"))
    out = torch.full_like(q, 3)
    rl.relibra_attention_fwd(q, k, v, zero[:1], out=out)      # no sequences
    assert torch.all(out == 3)
    rl.relibra_attention_fwd(q, k, v, zero, out=out)          # empty ones
    assert torch.all(out == 3)


@gpu
def test_attention_of_many_sequences():
    """More sequences than the scheduling block has threads, most of them a token or two."""
    g = torch.Generator().manual_seed(9)
    places = [int(x) for x in torch.randint(0, 4, (2500,), generator=g)]
    lens = [int(torch.randint(0, p + 1, (1,), generator=g)) for p in places]
    c = make(places, 1, 2, 32, lens=lens, seed=9)
    check(c, run(c))


@gpu
def test_attention_of_as_many_sequences_as_there_may_be():
    """8192 of one token each, and one more token's place of padding behind every second: a token's attention is its value."""
    n, d = 8192, 64
    g = torch.Generator().manual_seed(14)
    places = torch.tensor([1, 2] * (n // 2))
    start = torch.cat([torch.zeros(1, dtype=torch.long), places.cumsum(0)]).to(torch.int32)
    T = int(start[-1])
    q, k, v, do = (torch.randn(T, h, d, generator=g).to(BF16).to(DEV) for h in (2, 1, 1, 2))
    length = torch.ones(n, dtype=torch.int32, device=DEV)
    out, lse = rl.relibra_attention_fwd(q, k, v, start.to(DEV), seq_len=length)
    real = torch.zeros(T, dtype=torch.bool)
    real[start[:-1].long()] = True
    real = real.to(DEV)
    assert torch.equal(out[real], v[real].expand(-1, 2, -1)) and torch.all(out[~real] == 0) and torch.all(lse[~real] == 0)
    z = (q[real].double() * k[real].double()).sum(2) / 8
    assert torch.all((lse[real].double() - z).abs() <= (d + 12) * U * ((q[real].double() * k[real].double()).abs().sum(2) / 8 + z.abs()))
    dq, dk, dv = rl.relibra_attention_bwd(q, k, v, out, lse, do, start.to(DEV), seq_len=length)
    both = do[real].double().sum(1, keepdim=True)
    assert torch.all(dq == 0) and torch.all(dk == 0) and torch.all(dv[~real] == 0)
    assert torch.all((dv[real].double() - both).abs() <= H * both.abs() + 16 * U * do[real].double().abs().sum(1, keepdim=True))


@gpu
@pytest.mark.parametrize("places,lens,Hk,G", [([300, 129, 500], [300, 100, 481], 2, 4), ([2200, 200, 40], [2190, 100, 40], 1, 2)], ids=["short", "shared"])
def test_attention_in_a_graph_beside_eager_calls(places, lens, Hk, G):
    c = make(places, Hk, G, 128, lens=lens, seed=10)
    start, length = tables(c)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    ws = dict(f=rl.attention_fwd_workspace(c["T"], 3, Hk * G, Hk, 128), b=rl.attention_bwd_workspace(c["T"], 3, Hk * G, Hk, 128))
    flag = rl.new_err_flag()

    def step(q, f=None, b=None):
        out, lse = rl.relibra_attention_fwd(q, d["k"], d["v"], start, seq_len=length, workspace=f, err_flag=flag)
        return (out, lse, *rl.relibra_attention_bwd(q, d["k"], d["v"], out, lse, d["dout"], start, seq_len=length, workspace=b, err_flag=flag))
    step(d["q"], **ws)
    src = d["q"].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(src, **ws)
    side = torch.cuda.Stream()
    for turn in range(3):
        src.copy_(d["q"] * (turn + 1))
        length.copy_(torch.tensor([lens[0] - turn, lens[1] + turn, lens[2]], dtype=torch.int32))       # the schedule is made on the device
        want = step(src.clone())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = step(src)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want)), turn
    assert flag.item() == 0


@gpu
def test_attention_of_two_streams_at_once():
    """Calls that overlap, each with a workspace and a flag of its own, one of them with a table that is refused."""
    c = make([2100, 300], 1, 2, 128, seed=11)
    start, _ = tables(c)
    bad = torch.tensor([0, 1800, 1700], dtype=torch.int32, device=DEV)
    d = {n: c[n].to(DEV) for n in ("q", "k", "v", "dout")}
    flags = [rl.new_err_flag() for _ in range(2)]

    def step(table, flag):
        out, lse = torch.full((c["T"], 2, 128), 3.0, dtype=BF16, device=DEV), torch.full((c["T"], 2), 3.0, device=DEV)
        rl.relibra_attention_fwd(d["q"], d["k"], d["v"], table, out=out, lse=lse, err_flag=flag)
        grads = [torch.full((c["T"], h, 128), 3.0, dtype=BF16, device=DEV) for h in (2, 1, 1)]
        rl.relibra_attention_bwd(d["q"], d["k"], d["v"], out, lse, d["dout"], table, dq=grads[0], dk=grads[1], dv=grads[2], err_flag=flag)
        return (out, lse, *grads)
    want = step(start, flags[0])
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for s, table, flag in zip(side, (start, bad), flags):
            with torch.cuda.stream(s):
                got.append(step(table, flag))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x in got[::2] for a, b in zip(x, want)) and all(torch.all(a == 3) for x in got[1::2] for a in x)
    assert [f.item() for f in flags] == [0, rl.ERR_SEQ_TABLE]


@gpu
def test_attention_gradient_against_differences():
    """Central differences of the call's own output along random directions: T = 6 tokens, outputs in bf16."""
    c = make([6], 1, 2, 16, seed=11, peak=1.0)
    got = run(c)
    up = c["dout"].double()
    out_value = lambda cc: (run(cc, bwd=False)[0].cpu().double() * up).sum().item()
    g = torch.Generator().manual_seed(12)
    for name, grad in zip(("q", "k", "v"), got[2:]):
        way = torch.randn(c[name].shape, generator=g).sign().double() / 8              # steps that keep bf16's bits
        c1, c2 = (dict(c, **{name: (c[name].double() + s * way).to(BF16)}) for s in (1, -1))
        moved = (c1[name].double() - c2[name].double()) / 2
        slope = (moved * grad.cpu().double()).sum().item()
        # outputs are rounded (half a step of at most 4 each, twice) and p is; what the curve adds is the reference's own
        noise = 3 * H * (got[0].cpu().double().abs() * up.abs()).sum().item() + 2 * H * up.abs().sum().item()
        bend = abs(reference_value(c1, up) / 2 - reference_value(c2, up) / 2 - reference_slope(c, name, moved, up))
        tol = noise + bend + 4 * H * (moved.abs() * grad.cpu().double().abs()).sum().item() + 2 * H * up.abs().sum().item() * 0.5
        assert abs((out_value(c1) - out_value(c2)) / 2 - slope) <= tol


def bounds(c):
    """(errors of out, dq, dk, dv; the values themselves) of the sequences' tokens from the definition, by the tolerances at the top; zeros elsewhere."""
    T, Hk, G, d, s = c["T"], c["Hk"], c["G"], c["d"], c["scale"]
    z4 = lambda: [torch.zeros(T, h, d, dtype=torch.float64) for h in (Hk * G, Hk * G, Hk, Hk)]
    err, val = z4(), z4()
    for start, n in zip(c["starts"], c["lens"]):
        rows, mask = slice(start, start + n), torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(Hk):
            k, v = c["k"][rows, h].double(), c["v"][rows, h].double()
            for g in range(h * G, (h + 1) * G):
                q, do = c["q"][rows, g].double(), c["dout"][rows, g].double()
                z = (s * q @ k.T).masked_fill(~mask, -math.inf)
                ez = ((d + 4) * U * s * (q.abs() @ k.abs().T)).masked_fill(~mask, 0).amax(1, keepdim=True)
                lse = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - lse)
                want, size = p @ v, p @ v.abs()
                err_out = (H + 2 * ez + (2 * n + 40) * U) * size + H * want.abs()
                dp, D = do @ v.T, (do * want).sum(1, keepdim=True)
                ds = (p * (dp - D)).masked_fill(~mask, 0)
                ep = 2 * ez + (n + 32) * U + 8 * U * lse.abs()
                err_ds = (p * ((do.abs() * err_out).sum(1, keepdim=True) + (d + 8) * U * (do.abs() @ v.abs().T + (do.abs() * size).sum(1, keepdim=True))) + (2 * ep + H) * ds.abs()).masked_fill(~mask, 0)
                val[0][rows, g], err[0][rows, g] = want, err_out
                val[1][rows, g], err[1][rows, g] = s * ds @ k, s * (err_ds + (n + 24) * U * ds.abs()) @ k.abs()
                val[2][rows, h] += s * ds.T @ q
                val[3][rows, h] += p.T @ do
                err[2][rows, h] += s * (err_ds + (n * G + 24) * U * ds.abs()).T @ q.abs()
                err[3][rows, h] += ((H + ep + (n * G + 24) * U) * p).T @ do.abs()
    for i in (1, 2, 3):
        err[i] += H * val[i].abs()
    return err, val


STEPS = dict(q=1 / 4, k=1 / 4, v=1 / 4)


def differences(c, name, out_value):
    """(half the difference of `out_value` one step along the gradient's signs and one step back, how far it may be from the gradient's slope, the step, the definition's gradient).  Along the signs the
    slope is the sum of the gradient's sizes.  What the curve adds to a central difference is the definition's own."""
    i = ("q", "k", "v").index(name) + 1
    err, val = bounds(c)
    way = val[i].sign() * STEPS[name]
    c1, c2 = (dict(c, **{name: (c[name].double() + s * way).to(BF16)}) for s in (1, -1))
    moved = (c1[name].double() - c2[name].double()) / 2
    up = c["dout"].double()
    (e1, v1), (e2, v2) = bounds(c1), bounds(c2)
    slope = (moved * val[i]).sum().item()
    bend = abs(((v1[0] - v2[0]) * up).sum().item() / 2 - slope)
    tol = bend + ((e1[0] + e2[0]) * up.abs()).sum().item() / 2 + (moved.abs() * err[i]).sum().item()
    return (out_value(c1) - out_value(c2)) / 2, 1.01 * tol, moved, val[i]


DIFFERENCES = [dict(places=[6], Hk=1, G=2, d=16), dict(places=[40, 90], lens=[33, 90], Hk=2, G=1, d=64), dict(places=[70], Hk=1, G=5, d=72), dict(places=[150], Hk=1, G=2, d=128)]


def difference_case(kw):
    """Tokens of two kinds: their keys and values point one way or the other, beside something of their own; queries and the upstream ask for one kind, scores are about 1 and -1.  What a step
    changes then adds up over tokens and values, what is rounded does not."""
    c = make(**kw, seed=17, peak=1.0)
    g = torch.Generator().manual_seed(18)
    kind = torch.randn(c["T"], 1, 1, generator=g).sign()
    keys, values = (torch.randn(1, 1, c["d"], generator=g).sign() for _ in range(2))
    for n, way in (("q", keys), ("k", kind * keys), ("v", kind * values), ("dout", values)):
        c[n] = (way + 0.3 * c[n].float()).to(BF16)
    return dict(c, scale=1 / c["d"])


@gpu
@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("kw", DIFFERENCES, ids=str)
def test_attention_gradient_against_its_own_differences(kw, name):
    c = difference_case(kw)
    up = c["dout"].double()
    grad = run(c)[("q", "k", "v").index(name) + 2].cpu().double()
    diff, tol, moved, _ = differences(c, name, lambda cc: (run(cc, bwd=False)[0].cpu().double() * up).sum().item())
    assert abs(diff - (moved * grad).sum().item()) <= tol


@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("kw", DIFFERENCES, ids=str)
def test_attention_differences_tell_wrong_gradients(kw, name):
    """What the test above would say of other gradients, with the definition in the library's place: the right one passes; none, half of it, and one of the wrong sign do not,
    not even if everything that may be off were off in their favour."""
    c = difference_case(kw)
    diff, tol, moved, grad = differences(c, name, lambda cc: (bounds(cc)[1][0] * cc["dout"].double()).sum().item())
    right = (moved * grad).sum().item()
    assert abs(diff - right) <= tol
    for wrong in (0.0, 0.5, -1.0):
        assert abs(diff - wrong * right) > 2 * tol, (wrong, diff, right, tol)

def reference_out(q, k, v, s):
    kk, vv = k.repeat_interleave(q.shape[1] // k.shape[1], 1), v.repeat_interleave(q.shape[1] // k.shape[1], 1)
    z = torch.einsum("ihd,jhd->hij", q, kk) * s
    z = z.masked_fill(torch.ones(q.shape[0], q.shape[0], dtype=torch.bool).triu(1), -math.inf)
    return torch.einsum("hij,jhd->ihd", torch.softmax(z, 2), vv)


def reference_value(c, up):
    return (reference_out(c["q"].double(), c["k"].double(), c["v"].double(), c["scale"]) * up).sum().item()


def reference_slope(c, name, way, up):
    leaves = {n: c[n].double().requires_grad_(True) for n in ("q", "k", "v")}
    (reference_out(*leaves.values(), c["scale"]) * up).sum().backward()
    return (leaves[name].grad * way).sum().item()


@gpu
def test_attention_past_32_bits_of_offset():
    """Tokens 2^18 values apart: the last ones lie beyond 2^31 values (and 2^32 bytes) from the first."""
    T, stride = 9000, 1 << 18
    c = make([T - 300, 300], 1, 2, 64, seed=13)
    whole = torch.empty((T, stride), dtype=BF16, device=DEV)
    parts = [whole[:, a:a + h * 64].unflatten(1, (h, 64)) for a, h in ((0, 2), (128, 1), (192, 1), (256, 2), (384, 2), (512, 1), (576, 1), (640, 2))]
    for p, n in zip(parts, ("q", "k", "v", "dout")):
        p.copy_(c[n].to(DEV))
    want = run(c)
    start, _ = tables(c)
    out, lse = rl.relibra_attention_fwd(*parts[:3], start, out=parts[7])
    got = rl.relibra_attention_bwd(*parts[:3], out, lse, parts[3], start, dq=parts[4], dk=parts[5], dv=parts[6])
    assert all(torch.equal(a, b) for a, b in zip((out, lse, *got), want))
    # the short sequence at the far end, against the definition
    tail = slice(T - 300, T)
    short = dict(c, **{n: c[n][tail] for n in ("q", "k", "v", "dout")}, starts=[0, 300], lens=[300], T=300)
    check(short, [x[tail] for x in want])


# ------------------------------------------------------------------ refusals (no GPU needed: nothing is launched)
P, F, L = C.c_void_p, C.c_float, C.c_int64
M = 1 << 24


def _fwd(q=M, ql=256, k=2 * M, kl=128, v=3 * M, vl=128, start=4096, length=0, n_seq=2, T=8, Hq=4, Hk=2, d=64, scale=0.125, out=4 * M, ol=256, lse=4096, ws=4096, ws_bytes=1 << 40, flag=4096):
    return rl.lib().relibra_attention_fwd(P(q), L(ql), P(k), L(kl), P(v), L(vl), P(start), P(length), n_seq, T, Hq, Hk, d, F(scale), P(out), L(ol), P(lse), P(ws), C.c_size_t(ws_bytes), P(flag), P(0))


def _bwd(q=M, ql=256, k=2 * M, kl=128, v=3 * M, vl=128, start=4096, length=0, n_seq=2, T=8, Hq=4, Hk=2, d=64, scale=0.125, out=4 * M, ol=256, lse=4096, do=5 * M, dol=256, dq=6 * M, dql=256,
         dk=7 * M, dkl=128, dv=8 * M, dvl=128, ws=4096, ws_bytes=1 << 40, flag=4096):
    return rl.lib().relibra_attention_bwd(P(q), L(ql), P(k), L(kl), P(v), L(vl), P(out), L(ol), P(lse), P(do), L(dol), P(start), P(length), n_seq, T, Hq, Hk, d, F(scale), P(dq), L(dql), P(dk), L(dkl),
                                          P(dv), L(dvl), P(ws), C.c_size_t(ws_bytes), P(flag), P(0))


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_attention_refusals(call):
    for bad in (dict(T=-1), dict(n_seq=-1), dict(Hq=0), dict(Hk=0), dict(Hq=5), dict(d=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=0), dict(k=0),
                dict(v=0), dict(out=0), dict(lse=0), dict(start=0), dict(flag=0), dict(q=M + 2), dict(ql=248), dict(ql=260), dict(kl=(1 << 28) + 8), dict(ol=255), dict(ws=4104)):
        assert call(**bad) == rl.EINVAL, bad
    for bad in (dict(d=60), dict(d=136), dict(Hq=130), dict(Hq=8192, Hk=4096), dict(n_seq=8193), dict(T=(1 << 25) + 1)):
        assert call(**bad) == rl.EUNSUPPORTED, bad
    assert call(T=0, q=0, k=0, v=0, out=0) == rl.OK and call(n_seq=0, start=0) == rl.OK


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_attention_refuses_more_blocks_than_a_launch_has(call):
    """A launch has fewer than 2^32 threads, 256 a block; a block has 64 keys of a key head."""
    big = dict(Hq=64, Hk=64, d=8, ql=512, kl=512, vl=512, ol=512, n_seq=8192)
    assert call(T=1 << 24, **big) == rl.EUNSUPPORTED
    for which in (rl.WS_ATTENTION_FWD, rl.WS_ATTENTION_BWD):
        assert rl.workspace_bytes(which, 1 << 24, 1, 64, 8192, 64, 8) == 0 and rl.workspace_bytes(which, 1 << 23, 1, 64, 8192, 64, 8) > 0


def test_attention_refuses_overlaps_and_small_workspaces():
    for bad in (dict(out=M), dict(out=2 * M, ol=256), dict(out=3 * M + 16), dict(out=M + 256), dict(lse=4 * M + 64), dict(lse=M), dict(lse=3 * M - 64)):
        assert _fwd(**bad) == rl.EINVAL, bad
    for bad in (dict(do=0), dict(dq=0), dict(dk=0), dict(dv=0), dict(dol=255), dict(dq=M), dict(dq=4 * M), dict(dq=5 * M), dict(dk=2 * M), dict(dv=3 * M), dict(dk=8 * M), dict(dk=6 * M + 128), dict(lse=6 * M), dict(lse=8 * M - 4)):
        assert _bwd(**bad) == rl.EINVAL, bad
    for call, which in ((_fwd, rl.WS_ATTENTION_FWD), (_bwd, rl.WS_ATTENTION_BWD)):
        need = rl.workspace_bytes(which, 8, 1, 4, 2, 2, 64)
        assert need > 0 and call(ws_bytes=need - 1) == rl.EWORKSPACE and call(ws=0) == rl.EWORKSPACE
        assert rl.workspace_bytes(which, 8, 1, 4, 2, 3, 64) == 0 and rl.workspace_bytes(which, 8, 1, 4, 2, 2, 136) == 0


def test_attention_refuses_overlaps_of_tables_flag_and_workspace():
    """Outputs over the sequences' tables would change them while blocks find their work there.  Everything apart but for one pair."""
    small = {n: (100 + i) << 16 for i, n in enumerate(("start", "length", "lse", "flag", "ws"))}
    fwd_rows, bwd_rows = dict(q=M, k=2 * M, v=3 * M, out=4 * M), dict(q=M, k=2 * M, v=3 * M, out=4 * M, do=5 * M, dq=6 * M, dk=7 * M, dv=8 * M)
    for call, which, rows, outs, sums in ((_fwd, rl.WS_ATTENTION_FWD, fwd_rows, ("out",), ("lse", "ws", "flag")), (_bwd, rl.WS_ATTENTION_BWD, bwd_rows, ("dq", "dk", "dv"), ("ws", "flag"))):
        apart = dict(small, ws_bytes=rl.workspace_bytes(which, 8, 1, 4, 2, 2, 64))
        for name in (*outs, *sums):
            for other, at in {**small, **rows}.items():
                if other != name:
                    assert call(**{**apart, name: at}) == rl.EINVAL, (name, other)
        assert call(**{**apart, "flag": small["ws"] + apart["ws_bytes"] - 4}) == rl.EINVAL and call(**{**apart, "start": small["ws"] - 8}) == rl.EINVAL
        assert call(**{**apart, "length": rows[outs[0]] + 7 * 512 + 508}) == rl.EINVAL and call(**{**apart, "flag": rows["v"] + 4}) == rl.EINVAL


@gpu
def test_attention_takes_memory_between_its_rows():
    """lse, the tables and the flag in the gaps between the rows of the outputs: shared by no row, and left or written as they should be."""
    c = make([30, 25], 1, 2, 64, lens=[30, 20], seed=15)
    want = run(c)
    whole = torch.zeros((c["T"], 2048), dtype=BF16, device=DEV)
    out, dq, dk, dv = (whole[:, a:a + h * 64].unflatten(1, (h, 64)) for a, h in ((0, 2), (128, 2), (256, 1), (320, 1)))
    gap = lambda row, n, t: whole[row, 384:384 + 2 * n].view(t)
    start, length, flag, lse = gap(0, 3, torch.int32), gap(1, 2, torch.int32), gap(2, 1, torch.int32), gap(3, 110, torch.float32).view(55, 2)
    start.copy_(torch.tensor(c["starts"], dtype=torch.int32))
    length.copy_(torch.tensor(c["lens"], dtype=torch.int32))
    q, k, v, do = (c[n].to(DEV) for n in ("q", "k", "v", "dout"))
    rl.relibra_attention_fwd(q, k, v, start, seq_len=length, out=out, lse=lse, err_flag=flag)
    rl.relibra_attention_bwd(q, k, v, out, lse, do, start, seq_len=length, dq=dq, dk=dk, dv=dv, err_flag=flag)
    assert all(torch.equal(a, b) for a, b in zip((out, lse, dq, dk, dv), want)) and flag.item() == 0 and start.tolist() == c["starts"] and length.tolist() == c["lens"]

def test_attention_takes_interleaved_parts_of_one_tensor():
    """Refused for another reason (a workspace that is too small) behind the checks of overlaps: those let the parts pass."""
    kw = dict(q=M, k=M + 512, v=M + 768, ql=512, kl=512, vl=512)
    assert _fwd(**kw, ws_bytes=0) == rl.EWORKSPACE
    assert _bwd(**kw, dq=6 * M, dk=6 * M + 512, dv=6 * M + 768, dql=512, dkl=512, dvl=512, ws_bytes=0) == rl.EWORKSPACE
    assert _bwd(**kw, dq=6 * M, dk=6 * M + 256, dv=6 * M + 768, dql=512, dkl=512, dvl=512, ws_bytes=0) == rl.EINVAL
