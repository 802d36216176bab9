"""Log-probabilities of given tokens, entropies, alternatives and gradients against the fp64 oracle.

Tolerances.  A weight exp((z - m) / T) is a 32-bit power of two of y = (z - m) c, c = log2(e) / T rounded: three
roundings of y, |y| 2^-24 each, and the power's own, two steps of 2^-23 at most, so it is off by at most
delta(y) = 3 |y| 2^-24 + 2^-22 of itself (y in powers of two; ln 2 < 1).  Their sum's error relative to it is the mean of
delta under p, and so is the log's; sums of up to eight weights in 32 bits add 2^-21.  The entropy is the log less the
mean of ln 2 y, which is off by the mean of |y| delta and by the mean's share of the sum's error.  Results are rounded
to 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as O
from paper_2510_13847_amd import dynahead as D

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def tolerances(logp):
    """(of a log-probability, of the entropy) of a row, before the rounding of the results."""
    fine = logp[np.isfinite(logp)]
    if fine.size == 0:
        return 0.0, 0.0
    p = np.exp(fine)
    y = (fine.max() - fine) / math.log(2.0)
    delta = 3 * y * EPS + 2.0 ** -22
    mean = float((p * delta).sum()) + 2.0 ** -21
    return mean, mean + float((p * y * delta).sum()) + float((p * y).sum()) * mean


def check(logits, tokens, temperature, top, got, names=None, lengths=None):
    """Every row of a call against the oracle."""
    z = logits.double().cpu().numpy()
    tk = tokens.cpu().numpy().reshape(z.shape[0], -1)
    lp = got.logprobs.cpu().double().numpy().reshape(tk.shape)
    entropy = got.entropy.cpu().double().numpy()
    for r in range(z.shape[0]):
        n = z.shape[1] if lengths is None else int(lengths[r])
        who = range(n) if names is None else names[r][:n]
        given, h, best, logp = O.token_logprobs(z[r, :n], who, tk[r], temperature, top)
        a, b = tolerances(logp)
        same(lp[r], given, a)
        same(entropy[r:r + 1], np.array([h]), b)
        if top:
            assert got.top_ids[r].tolist() == [i for i, _ in best], r
            same(got.top_logprobs[r].cpu().double().numpy(), np.array([x for _, x in best]), a)
        if got.stats is not None and n and np.isfinite(logp).any():
            assert float(got.stats[r, 0]) == z[r, :n].max()


def same(got, want, tol):
    assert np.array_equal(np.isnan(got), np.isnan(want)), (got, want)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), (got, want)
    off = np.abs(got[fine] - want[fine])
    assert (off <= tol + EPS * np.abs(want[fine])).all(), (off.max(), tol)


def rows(N, V, dtype, seed, pad=0, lead=0, scale=3.0):
    base = torch.full((lead + N * (V + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    z = base[lead:].as_strided((N, V), (V + pad, 1))
    z.copy_((torch.randn((N, V), generator=gen(seed)) * scale).to(DT[dtype]))
    return z


def some_tokens(N, V, T, seed):
    """Tokens of the row, ids outside it and repeats."""
    t = torch.randint(0, V, (N, T), generator=gen(seed))
    kind = torch.randint(0, 12, (N, T), generator=gen(seed + 1))
    t[kind == 0] = -1
    t[kind == 1] = V
    t[kind == 2] = 2 ** 31 - 1
    if T > 1:
        t[:, T - 1] = t[:, 0]
    return t.to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,T,top,pad,lead", [(1, 1, 1, 1, 0, 0), (2, 2, 2, 3, 1, 1), (3, 7, 1, 8, 0, 3), (5, 64, 3, 64, 3, 0),
                                                (4, 255, 2, 5, 0, 1), (3, 2047, 1, 20, 1, 5), (3, 2048, 0, 10, 0, 0),
                                                (2, 2049, 64, 64, 7, 2), (7, 8191, 4, 1, 0, 0), (2, 8193, 1, 0, 2, 1),
                                                (3, 50021, 2, 33, 1, 0), (1, 128256, 1, 10, 0, 0), (2, 151936, 3, 64, 0, 0),
                                                (1, 262144, 2, 7, 0, 0), (300, 513, 1, 4, 0, 0), (1100, 40, 2, 6, 3, 0),
                                                (600, 5000, 1, 16, 1, 0)])
def test_logprobs(N, V, T, top, pad, lead, dtype):
    z = rows(N, V, dtype, N + V, pad, lead)
    t = some_tokens(N, V, T, V)
    check(z, t, 1.0, top, D.token_logprobs(z, t, top=top, want_stats=True))


@pytest.mark.parametrize("temperature", [0.0625, 0.7, 5.0, 1e-3, 1e4, 1.2e-38, 2.9e38])
def test_temperatures(temperature):
    temperature = float(np.float32(temperature))
    z = rows(3, 1000, "f32", 1)
    z[2] = z[2].round()  # equal largest logits
    t = some_tokens(3, 1000, 4, 2)
    got = D.token_logprobs(z, t, temperature=temperature, top=5)
    if temperature > 1e-30:
        check(z, t, temperature, 5, got)
    else:  # log-probabilities past 32 bits are -inf
        assert got.top_ids[0, 0] == z[0].argmax() and (got.logprobs <= 0).all() and float(got.entropy[0]) == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 3000, 20000])
def test_masks_and_undefined_logits(V, dtype):
    inf = float("inf")
    low = torch.finfo(DT[dtype]).min
    z = rows(13, V, dtype, V)
    z[0] = -inf                                   # nothing is allowed
    z[1] = low                                    # masked by the lowest number throughout: uniform
    z[2, torch.rand(V, generator=gen(1)) < 0.9] = -inf
    z[3, torch.rand(V, generator=gen(2)) < 0.9] = low
    z[4] = -inf
    z[4, V - 1] = 0.25                            # one token left
    z[5, V // 2] = float("nan")
    z[6, V // 3] = inf
    z[7] = float("nan")
    z[8] = torch.finfo(DT[dtype]).max             # uniform at the other end
    z[9] = -inf
    z[9, 0], z[9, V - 1] = low, low               # two tokens at the lowest number
    z[10] = 0.0
    z[10, ::2] = -0.0                             # zeros of both signs are equal
    z[11, 5], z[11, 6] = inf, -inf
    z[12] = -inf
    z[12, 3] = float("nan")
    t = torch.tensor([[0, V - 1, V // 2, -1]], dtype=torch.int32).expand(13, 4).contiguous().cuda()
    got = D.token_logprobs(z, t, top=min(12, V), want_stats=True)
    check(z, t, 1.0, min(12, V), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_that_begin_late_in_long_rows(dtype):
    """Masked logits met by some threads only, from the first, second or last columns on, in rows of one workgroup each."""
    V, N = 40000, 1040
    z = rows(8, V, dtype, 3)
    z[0, 9000] = -float("inf")
    z[1, 20000:] = -float("inf")
    z[2, V - 1] = -float("inf")
    z[3, :30000] = -float("inf")
    z[4, 8192 * 2:8192 * 3] = -float("inf")
    z[5, 17000::2048] = -float("inf")
    z[6, 9000] = float("nan")
    z[7, 8192 * 4:] = -float("inf")
    t = torch.tensor([[0, 9000, 20001, V - 1]], dtype=torch.int32).expand(8, 4).contiguous().cuda()
    for temperature in (1.0, 1e-7):  # the second with its weights by the difference
        got = D.token_logprobs(z.repeat(N // 8, 1), t.repeat(N // 8, 1), temperature=temperature, top=10)
        for name in ("logprobs", "entropy", "top_ids", "top_logprobs"):
            x = getattr(got, name)
            first = x[:8].repeat(N // 8, *[1] * (x.dim() - 1))
            assert torch.equal(torch.nan_to_num(x.double(), nan=7.0), torch.nan_to_num(first.double(), nan=7.0))
            setattr(got, name, x[:8])
        if temperature == 1.0:
            check(z, t, 1.0, 10, got)
        else:  # the largest logit has all the weight, shared where several have it
            best = z.float().max(1).values
            assert torch.equal(got.top_logprobs[:, 0].isnan().cpu(), torch.tensor([r == 6 for r in range(8)]))
            for r in (0, 1, 2, 3, 4, 5, 7):
                many = int((z[r].float() == best[r]).sum())
                assert abs(float(got.top_logprobs[r, 0]) + math.log(many)) <= 2.0 ** -18
                assert abs(float(got.entropy[r]) - math.log(many)) <= 2.0 ** -18


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 9000, 70000])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "steps", "ends"])
def test_alternatives_of_rows_with_many_equal_or_sorted_logits(kind, V, dtype):
    i = torch.arange(V)
    z = {"equal": torch.ones(V), "rising": i / 256.0, "falling": -i / 256.0, "two": (i % 2).float(),
         "steps": (i * 7 // 1000).float() % 5, "ends": ((i < 20) | (i >= V - 20)).float() * (1 + i % 3)}[kind]
    z = z.to(DT[dtype])[None].cuda()
    for top in (1, 20, 64):
        t = torch.tensor([[0, V - 1]], dtype=torch.int32).cuda()
        check(z, t, 1.0, top, D.token_logprobs(z, t, top=top))


@pytest.mark.parametrize("kind", ["equal", "rising", "two", "late"])
def test_many_rows_with_many_equal_or_sorted_logits(kind):
    """Rows that one workgroup goes through in several sweeps, the list not empty when a sweep overflows it."""
    V = 30000
    i = torch.arange(V)
    z = {"equal": torch.ones(V), "rising": i / 8.0, "two": (i % 2).float(),
         "late": torch.where(i < 20000, torch.randn(V, generator=gen(1)), torch.full((V,), 9.0))}[kind]
    z = z.float()[None].expand(1030, V).contiguous().cuda()
    t = torch.full((1030, 1), 5, dtype=torch.int32).cuda()
    for top in (1, 20, 64):
        got = D.token_logprobs(z, t, top=top)
        for x in (got.logprobs, got.entropy, got.top_ids, got.top_logprobs):
            assert torch.equal(x, x[:1].expand_as(x))
        for name in ("logprobs", "entropy", "top_ids", "top_logprobs"):
            setattr(got, name, getattr(got, name)[:1])
        check(z[:1], t[:1], 1.0, top, got)


# ---------------------------------------------------------------- shortlists
def shortlists(V, M, k, N, seed, dtype="f32"):
    g = gen(seed)
    of = torch.randint(0, M, (V,), generator=g)
    of[of == M // 2] = 0  # an empty cluster
    layout = D.build_layout(of.to(torch.int32).cuda(), torch.zeros((V, 8), device="cuda"), M)
    clusters = torch.stack([torch.randperm(M, generator=g)[:k] for _ in range(N)]).to(torch.int32)
    clusters[0, 0] = M // 2
    if N > 2:
        clusters[1, :] = M // 2  # an empty shortlist
        clusters[2, k // 2:] = -1
    sel, off, length, ids = D.shortlist(layout, clusters.cuda())
    z = torch.full(ids.shape, float("nan"), dtype=DT[dtype], device="cuda")
    for r in range(N):
        z[r, :int(length[r])] = (torch.randn(int(length[r]), generator=g) * 3).to(DT[dtype])
    return layout, (sel, off, length), ids.cpu().numpy(), z, [int(n) for n in length]


@pytest.mark.parametrize("V,M,k,N,T,top", [(100, 5, 2, 4, 3, 7), (3000, 64, 8, 9, 2, 20), (50000, 100, 40, 5, 5, 64),
                                           (2000, 30, 30, 3, 1, 10), (8191, 2000, 300, 3, 4, 5), (50, 50, 1, 4, 2, 3),
                                           (9001, 2000, 700, 4, 3, 64), (30000, 1500, 1500, 5, 4, 20)])
def test_shortlists(V, M, k, N, T, top):
    layout, sel, ids, z, length = shortlists(V, M, k, N, V + k)
    # half of the tokens from the row's own
    t = some_tokens(N, V, T, k)
    for r in range(N):
        if length[r]:
            t[r, 0] = int(ids[r, (7 * r) % length[r]])
    where = D.ShortlistRows(layout, *sel)
    got = D.token_logprobs(z, t, temperature=0.8, top=top, rows=where, want_stats=True)
    check(z, t, float(np.float32(0.8)), top, got, ids, length)
    # equal logits: by token, not by slot
    z[:, :] = 1.0
    check(z, t, 1.0, top, D.token_logprobs(z, t, top=top, rows=where), ids, length)


def test_rows_that_share_a_shortlist():
    layout, _, _, _, _ = shortlists(2000, 40, 6, 3, 1)
    sel, off, length, ids = D.shortlist(layout, torch.tensor([[3, 9, 9, 31, -1, 4]], dtype=torch.int32).cuda())
    n = int(length[0])
    z = torch.randn((5, n + 4), generator=gen(3)).cuda()
    t = ids[0, torch.randint(0, n, (5,), generator=gen(4)).cuda()].contiguous()
    got = D.token_logprobs(z, t, top=4, rows=D.ShortlistRows(layout, sel, off, length))
    names = ids.cpu().numpy().repeat(5, 0)
    check(z, t, 1.0, 4, got, names, [n] * 5)


# ---------------------------------------------------------------- gradients
def gradient_check(z, t, g, e, temperature, stats_of, grad, names=None, lengths=None):
    zz, tt = z.double().cpu().numpy(), t.cpu().numpy().reshape(z.shape[0], -1)
    gg = g.double().cpu().numpy().reshape(tt.shape)
    got = grad.double().cpu().numpy()
    half = torch.finfo(grad.dtype).eps / 2
    for r in range(z.shape[0]):
        n = z.shape[1] if lengths is None else int(lengths[r])
        who = list(range(n)) if names is None else [int(x) for x in names[r][:n]]
        ee = 0.0 if e is None else float(e[r])
        want = O.token_logprobs_grad(zz[r, :n], who, tt[r], gg[r], ee, temperature)
        _, h, _, logp = O.token_logprobs(zz[r, :n], who, [], temperature)
        assert np.array_equal(np.isnan(got[r, :n]), np.isnan(want))
        p = np.nan_to_num(np.exp(logp))
        lp = np.where(np.isfinite(logp), logp, 0.0)
        mine = [w for x, w in zip(tt[r], gg[r]) if x in set(who)]
        size = np.abs(sum(mine)) * p + abs(ee) * p * (np.abs(lp) + abs(np.nan_to_num(h)))
        # p as above, a few more roundings of its factors, and the sum of a token's own terms
        tol = size * ((np.abs(lp) * 6 + 16) * EPS) / temperature + abs(ee) * p * (np.abs(lp) + 1) * 8 * EPS / temperature
        tol += sum(abs(w) for w in mine) * 4 * EPS / temperature * np.isin(who, tt[r])
        off = np.abs(got[r, :n] - want)
        bound = tol + half * (np.abs(want) + tol) + np.finfo(np.float32).tiny
        assert (off[~np.isnan(want)] <= bound[~np.isnan(want)]).all(), (r, np.nanmax(off / bound))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,T,pad,lead,temperature", [(1, 1, 1, 0, 0, 1.0), (3, 7, 2, 1, 1, 0.5), (4, 100, 3, 0, 3, 1.0),
                                                        (2, 2047, 1, 3, 0, 2.0), (3, 2049, 64, 0, 1, 1.0),
                                                        (5, 8191, 4, 1, 0, 0.75), (2, 70001, 2, 0, 0, 1.0),
                                                        (2, 131072, 5, 0, 0, 1.0), (400, 600, 1, 0, 0, 1.0)])
def test_gradients(N, V, T, pad, lead, temperature, dtype):
    z = rows(N, V, dtype, V + 1, pad, lead)
    t = some_tokens(N, V, T, V)
    g, e = torch.randn((N, T), generator=gen(5)).cuda(), torch.randn(N, generator=gen(6)).cuda()
    if N > 2:
        g[1], e[1] = 0.0, 0.0  # padding
        e[2] = 0.0
    stats = D.token_logprobs(z, t, temperature=temperature, want_stats=True).stats
    base = torch.full((lead + N * (V + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    out = base[lead:].as_strided((N, V), (V + pad, 1))
    for ee in (e, None):
        base.fill_(float("nan"))
        grad = D.token_logprobs_grad(z, stats, t, g, ee, temperature=temperature, out=out)
        gradient_check(z, t, g, ee, temperature, stats, grad)
        assert int(torch.isnan(base).sum()) == base.numel() - N * V
    fresh = D.token_logprobs_grad(z, stats, t, g, None, temperature=temperature)
    assert torch.equal(fresh, out)


@pytest.mark.parametrize("temperature", [1.2e-38, 1e-20, 1e20, 2.9e38])
def test_gradients_at_the_ends_of_temperatures(temperature):
    """All weight on the largest logit, or evenly spread: the gradient is the given tokens' own, or that less a share."""
    temperature = float(np.float32(temperature))
    z = rows(2, 500, "f32", 4)
    best = z.argmax(1).to(torch.int32)
    t = torch.stack([best, (best + 1) % 500], 1).contiguous()
    g = torch.tensor([[0.5, 0.0], [0.25, 0.25]]).cuda()
    e = torch.tensor([3.0, 0.0]).cuda()
    stats = D.token_logprobs(z, t, temperature=temperature, want_stats=True).stats
    grad = D.token_logprobs_grad(z, stats, t, g, e, temperature=temperature).double().cpu()
    want = torch.zeros((2, 500), dtype=torch.float64)
    share = 0.0 if temperature < 1.0 else 1.0 / 500
    for r in range(2):
        want[r] -= share * 0.5
        if temperature < 1.0:
            want[r, int(best[r])] -= 0.5
        want[r, int(t[r, 0])] += float(g[r, 0])
        want[r, int(t[r, 1])] += float(g[r, 1])
    want /= temperature
    # past 32 bits nothing is left of it; a share is off by a few steps and by exp(z / T) - 1 < 1e-18
    assert torch.isfinite(grad).all()
    assert ((grad - want).abs() <= 2.0 ** -20 * 0.5 / temperature + 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_masked_rows(dtype):
    inf, V = float("inf"), 3000
    low = torch.finfo(DT[dtype]).min
    z = rows(9, V, dtype, 1)
    z[8] = float("nan")
    z[0] = -inf
    z[1] = low
    z[2, torch.rand(V, generator=gen(1)) < 0.9] = -inf
    z[2, 5] = -inf                     # a given token that is masked
    z[3, torch.rand(V, generator=gen(2)) < 0.9] = low
    z[4] = -inf
    z[4, 7] = 1.0
    z[5, 9] = float("nan")
    z[6, 9] = inf
    z[7, 11] = float("nan")            # in a padding row, which nothing reads
    t = torch.tensor([[5, 7, 5, -1]], dtype=torch.int32).expand(9, 4).contiguous().cuda()
    g, e = torch.randn((9, 4), generator=gen(3)).cuda(), torch.randn(9, generator=gen(4)).cuda()
    g[7], e[7] = 0.0, 0.0
    g[7, 3] = 5.0                      # at a token that is not there: not used
    g[:, 3] = float("nan")
    stats = D.token_logprobs(z, t, want_stats=True).stats
    grad = D.token_logprobs_grad(z, stats, t, g, e)
    assert (grad[0] == 0).all() and (grad[7] == 0).all()
    assert torch.isnan(grad[5]).all() and torch.isnan(grad[6]).all() and torch.isnan(grad[8]).all()
    keep = [0, 1, 2, 3, 4, 7]
    gradient_check(z[keep], t[keep], g[keep], e[keep], 1.0, stats[keep], grad[keep])


def test_gradient_of_shortlists():
    layout, sel, ids, z, length = shortlists(5000, 50, 9, 6, 2)
    t = some_tokens(6, 5000, 3, 1)
    for r in range(6):
        if length[r]:
            t[r, 0] = int(ids[r, length[r] // 2])
    g, e = torch.randn((6, 3), generator=gen(3)).cuda(), torch.randn(6, generator=gen(4)).cuda()
    where = D.ShortlistRows(layout, *sel)
    stats = D.token_logprobs(z, t, rows=where, want_stats=True).stats
    out = torch.full_like(z, 7.0)
    D.token_logprobs_grad(z, stats, t, g, e, rows=where, out=out)
    gradient_check(z, t, g, e, 1.0, stats, out, ids, length)
    for r in range(6):
        assert (out[r, length[r]:] == 7.0).all()
    assert torch.equal(D.token_logprobs_grad(z, stats, t, g, e, rows=where)[0, :length[0]], out[0, :length[0]])


def test_gradient_against_differences():
    """The objective's own differences: z moves by h, a power of two; its third derivative is below 10 here, and the
    forward results' tolerance is divided by 2 h."""
    V = 37
    z = rows(1, V, "f32", 3, scale=1.0)
    t = torch.tensor([[3, 20, 3]], dtype=torch.int32).cuda()
    g, e = torch.tensor([[0.5, -1.0, 0.25]]).cuda(), torch.tensor([0.75]).cuda()

    def objective(x):
        r = D.token_logprobs(x, t)
        return float((g.double() * r.logprobs.double()).sum() + (e.double() * r.entropy.double()).sum())

    grad = D.token_logprobs_grad(z, D.token_logprobs(z, t, want_stats=True).stats, t, g, e)
    h = 2.0 ** -5
    for i in range(V):
        up, down = z.clone(), z.clone()
        up[0, i] += h
        down[0, i] -= h
        step = float(up[0, i].double() - down[0, i].double())
        assert abs((objective(up) - objective(down)) / step - float(grad[0, i])) < 10 * h * h / 6 + 4e-6 / h


# ---------------------------------------------------------------- long rows, streams, graphs
def test_offsets_past_32_bits():
    """Rows that start past 2^31 elements."""
    V, stride = 1 << 20, (1 << 30) + 3
    base = torch.empty(4 * stride + 2 * V, dtype=torch.bfloat16, device="cuda")
    z = base.as_strided((5, V), (stride, 1))
    small = (torch.randn((5, V), generator=gen(1)) * 3).to(torch.bfloat16)
    z.copy_(small)
    t = torch.tensor([[0], [V - 1], [7], [V // 2], [V - 2]], dtype=torch.int32).cuda()
    got = D.token_logprobs(z, t, top=3, want_stats=True)
    ref = D.token_logprobs(small.cuda(), t, top=3, want_stats=True)
    for a, b in ((got.logprobs, ref.logprobs), (got.entropy, ref.entropy), (got.top_ids, ref.top_ids), (got.stats, ref.stats)):
        assert torch.equal(a, b)
    g = torch.ones((5, 1), device="cuda")
    out = base[V:]  # beside the logits, in the same rows' gaps: their spans overlap
    with pytest.raises(D.DynaError):
        D.token_logprobs_grad(z, got.stats, t, g, out=out.as_strided((5, V), (stride, 1)))
    apart = torch.empty(4 * stride + V, dtype=torch.bfloat16, device="cuda").as_strided((5, V), (stride, 1))
    assert torch.equal(D.token_logprobs_grad(z, got.stats, t, g, out=apart),
                       D.token_logprobs_grad(small.cuda(), got.stats, t, g))


@pytest.mark.parametrize("N", [2, 700])
def test_another_stream(N):
    z = rows(N, 5000, "bf16", 1)
    t = some_tokens(N, 5000, 2, 3)
    want = D.token_logprobs(z, t, top=4, want_stats=True)
    g = torch.randn((N, 2), generator=gen(4)).cuda()
    grad = D.token_logprobs_grad(z, want.stats, t, g)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = D.token_logprobs(z, t, top=4, want_stats=True, stream=s)
    other = D.token_logprobs_grad(z, got.stats, t, g, stream=s)
    s.synchronize()
    assert torch.equal(got.logprobs, want.logprobs) and torch.equal(got.top_ids, want.top_ids) and torch.equal(other, grad)


@pytest.mark.parametrize("N", [2, 700])
def test_captured_and_replayed(N):
    """Two captured graphs with a workspace each, replayed in turn on new logits, with eager calls between."""
    V = 6000
    z, t = rows(N, V, "bf16", 1), some_tokens(N, V, 2, 3)
    g = torch.randn((N, 2), generator=gen(4)).cuda()
    D.token_logprobs(z, t, top=5)
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        ws = D.token_logprobs_workspace(N, V, 2, 5)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = D.token_logprobs(z, t, top=5, want_stats=True, ws=ws)
            d = D.token_logprobs_grad(z, r.stats, t, g)
        graphs.append((graph, ws))
        results.append((r, d))
    for seed in range(5, 9):
        z.copy_((torch.randn((N, V), generator=gen(seed)) * 3).to(z.dtype))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = D.token_logprobs(z, t, top=5, want_stats=True)
        grad = D.token_logprobs_grad(z, want.stats, t, g)
        for r, d in results:
            assert torch.equal(r.logprobs, want.logprobs) and torch.equal(r.entropy, want.entropy)
            assert torch.equal(r.top_ids, want.top_ids) and torch.equal(d, grad)


def test_one_dimension_of_tokens_and_no_rows():
    z = rows(6, 300, "f32", 1)
    t = some_tokens(6, 300, 1, 2)
    a, b = D.token_logprobs(z, t), D.token_logprobs(z, t[:, 0].contiguous())
    assert a.logprobs.shape == (6, 1) and b.logprobs.shape == (6,) and torch.equal(a.logprobs[:, 0], b.logprobs)
    assert D.token_logprobs(z[:0], t[:0], top=3).top_ids.shape == (0, 3)


def test_binding_refuses():
    z, t = rows(4, 100, "f32", 1), some_tokens(4, 100, 2, 2)
    for bad in (dict(tokens=t.long()), dict(logits=z.half())):
        with pytest.raises(TypeError):
            D.token_logprobs(**dict(dict(logits=z, tokens=t), **bad))
    for bad in (dict(tokens=t[:3]), dict(tokens=t.t()), dict(logits=z.t())):
        with pytest.raises(ValueError):
            D.token_logprobs(**dict(dict(logits=z, tokens=t), **bad))
    for bad in (dict(top=65), dict(temperature=0.0), dict(ws=torch.zeros(1, dtype=torch.uint8, device="cuda")[:0])):
        with pytest.raises(D.DynaError):
            D.token_logprobs(z, t, **bad)
    layout, sel, ids, zs, length = shortlists(100, 5, 2, 3, 1)
    with pytest.raises(ValueError):
        D.token_logprobs(z, t, rows=D.ShortlistRows(layout, *sel))
    with pytest.raises(ValueError):
        D.ShortlistRows(layout, sel[0], sel[0], sel[2])
    r = D.token_logprobs(z, t, want_stats=True)
    with pytest.raises(ValueError):
        D.token_logprobs_grad(z, r.stats[:, :2], t, torch.zeros((4, 2), device="cuda"))
    with pytest.raises(D.DynaError):
        D.token_logprobs_grad(z, r.stats, t, torch.zeros((4, 2), device="cuda"), out=z)
