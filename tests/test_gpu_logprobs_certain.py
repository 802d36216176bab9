"""Rows whose largest logit has almost all of the weight: log p of it is -log(1 + r), where r is what the others weigh,
and the entropy is as small, so both are held to a share of themselves.

Tolerances.  With y = (z - m) log2(e) / T, an other token's weight 2^y is off by delta = 4 |y| 2^-24 + 2^-22 of itself
(c = log2(e) / T rounded, the product's and the difference's rounding, the rescaling's; the power's two steps of 2^-23),
sums of 32 by 2^-21 and a row's rescalings by 2^-22 a sweep of 8192 columns.  r is off by the mean of that under the
others' weights.  The entropy is log(1 + r) and the mean of |y|, each of whose terms is off by another 2^-23.  Weights
below 2^-125 may be lost.  The largest logit's own weight is 1 and adds nothing up to r = 1/2; beyond, it is a weight
like the others, off by 2^-22 and its sum's 2^-21, over 1 + r.  The row's sums are 64-bit numbers that hold the largest
weight, 1, until it is taken out again: each of their additions since (one a sweep, 16 at most, six and four where
threads and waves are joined, as many where parts are, and one to take it out: 37, less than 64) is off by 2^-53, in
what the others weigh and, with log2 of a weight below 75 where that counts, in the entropy.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2510_13847_amd import dynahead as D

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 2.0 ** -24


def exact_row(z, T):
    """(place of the largest logit, r, log-probabilities, entropy, share of r that may be wrong, of the mean of |y|)."""
    best = int(z.argmax())
    y = (z - z[best]) / T
    w = np.exp(y)
    w[best] = 0.0
    r = float(w.sum())
    mean = float(-(w[w > 0] * y[w > 0]).sum())
    logp = y - math.log1p(r)
    two = np.abs(y) / math.log(2.0)
    steps = 2.0 ** -21 + 2.0 ** -22 * -(-len(z) // 8192)
    off_r = float((w[w > 0] * (4 * two[w > 0] * EPS + 2.0 ** -22)).sum()) / max(r, 1e-300) + steps
    off_y = float((w * np.where(w > 0, np.abs(y), 0.0))[w > 0] @ (4 * two[w > 0] * EPS + 2.0 ** -22 + 2.0 ** -23)) / max(mean, 1e-300) + steps
    return best, r, logp, math.log1p(r) + mean / (1.0 + r), off_r, off_y


def log_s_tolerance(r, off_r, V):
    own = (2.0 ** -22 + 2.0 ** -21) / (1.0 + r) if r > 0.499 else 0.0
    return off_r * math.log1p(r) + own + 64 * 2.0 ** -53 + V * 2.0 ** -125


def certain_rows(V, dtype, seed, lift=0.0, gaps=(0.0, 1.0, 3.0, 6.0, 9.0, 12.0, 20.0, 60.0)):
    """A row for each power of ten by which its largest logit outweighs the others."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((len(gaps), V), generator=g) * 0.75
    at = torch.randint(0, V, (len(gaps),), generator=g)
    for r, gap in enumerate(gaps):
        z[r, at[r]] = math.log(V * 10.0 ** gap) + 1.0
    return (z + lift).to(DT[dtype])


def check_row(z, T, given, entropy, tokens):
    best, r, logp, H, off_r, off_y = exact_row(z, T)
    off, log_s = log_s_tolerance(r, off_r, len(z)), math.log1p(r)
    for token, got in zip(tokens, given):
        want = logp[token]
        assert got <= 0.0
        assert abs(got - want) <= off + EPS * abs(want), (token == best, got, want)
    assert entropy >= 0.0
    # (200: |y| of a lost weight that counts)
    assert abs(entropy - H) <= off + (off_y + off_r + off) * (H - log_s) + EPS * H + 200 * len(z) * 2.0 ** -125, (entropy, H)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,N", [(1, 8), (2, 8), (33, 8), (2049, 8), (8200, 8), (30000, 8), (128256, 8), (300, 1040),
                                 (20001, 1040)])
@pytest.mark.parametrize("temperature,lift", [(1.0, 0.0), (0.7, -25.0), (1.0, 300.0), (3.0, 5.0)])
def test_rows_of_one_likely_token(V, N, dtype, temperature, lift):
    T = float(np.float32(temperature))
    z = certain_rows(V, dtype, V, lift)
    best = z.double().argmax(1)
    tokens = torch.stack([best, (best + 1) % V, torch.full_like(best, V - 1)], 1).to(torch.int32)
    top = min(3, V)
    got = D.token_logprobs(z.repeat(N // 8, 1).cuda(), tokens.repeat(N // 8, 1).cuda(), temperature=T, top=top, want_stats=True)
    for name in ("logprobs", "entropy", "top_ids", "top_logprobs", "stats"):
        x = getattr(got, name)
        assert torch.equal(x, x[:8].repeat(N // 8, *[1] * (x.dim() - 1)))
    for r in range(8):
        zz = z[r].double().numpy()
        if V > 1 and (zz == zz.max()).sum() > 1:
            continue  # rounding the row to the type made two of them
        check_row(zz, T, got.logprobs[r].double().tolist(), float(got.entropy[r]), tokens[r].tolist())
        assert float(got.top_logprobs[r, 0]) == float(got.logprobs[r, 0]) and int(got.top_ids[r, 0]) == int(best[r])
        # what the gradient takes
        assert float(got.stats[r, 0]) == zz.max()
        _, rest, _, H, off_r, off_y = exact_row(zz, T)
        assert abs(float(got.stats[r, 1]) - math.log1p(rest)) <= log_s_tolerance(rest, off_r, V)


@pytest.mark.parametrize("N", [3, 1041])
def test_weights_by_the_difference(N):
    """Logits over a temperature that puts their powers past 2^20: one step of the type is a third of a power of two."""
    V, T = 20000, 2.0 ** -20
    steps = torch.randint(40, 400, (3, V), generator=torch.Generator().manual_seed(1))
    steps[0, 77], steps[1, 19999], steps[2, 0] = 0, 0, 0
    z = 1.875 - steps.float() * 2.0 ** -22
    tokens = torch.tensor([[77, 5], [19999, 5], [0, 5]], dtype=torch.int32)
    got = D.token_logprobs(z.repeat(N // 3, 1).cuda(), tokens.repeat(N // 3, 1).cuda(), temperature=T)
    for r in range(3):
        check_row(z[r].double().numpy(), T, got.logprobs[r].double().tolist(), float(got.entropy[r]), tokens[r].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_others_masked_or_far(dtype):
    """Nothing but the largest logit: log p and entropy are 0; one other far below it among masked ones."""
    inf, low = float("inf"), torch.finfo(DT[dtype]).min
    for V in (40, 20000):
        z = torch.full((5, V), -inf)
        z[0, 3] = 7.25
        z[1], z[1, V - 1] = low, -2.5
        z[2, 9], z[2, 10] = 30.0, 12.0
        z[3, V - 1], z[3, 0] = -40.0, -61.0
        z[4, 5], z[4, V - 2] = 100.5, 100.0  # no such row: about 0.62 and 0.38
        tokens = torch.tensor([[3, 0], [V - 1, 0], [9, 10], [V - 1, 0], [5, V - 2]], dtype=torch.int32)
        got = D.token_logprobs(z.to(DT[dtype]).cuda(), tokens.cuda())
        for r in (0, 1):
            assert float(got.logprobs[r, 0]) == 0.0 and float(got.entropy[r]) == 0.0
        for r, gap in ((2, 18.0), (3, 21.0), (4, 0.5)):
            rest = math.exp(-gap)
            off = 2.0 ** -19 + 4 * gap * 1.5 * EPS
            assert abs(float(got.logprobs[r, 0]) + math.log1p(rest)) <= off * math.log1p(rest)
            assert abs(float(got.logprobs[r, 1]) + gap + math.log1p(rest)) <= off * math.log1p(rest) + EPS * (gap + 1)
            H = math.log1p(rest) + gap * rest / (1.0 + rest)
            assert abs(float(got.entropy[r]) - H) <= 2 * off * H


@pytest.mark.parametrize("N", [2, 1040])
def test_two_equal_logits_at_the_top(N):
    """Two halves, however the columns fall to threads, sweeps and parts."""
    V = 30000
    for a, b in ((0, 1), (0, 8), (5, 2048 + 5), (3, 8192 + 3), (100, 29999)):
        z = torch.full((N, V), -90.0)
        z[:, a], z[:, b] = 50.0, 50.0
        got = D.token_logprobs(z.cuda(), torch.tensor([[a, b]], dtype=torch.int32).expand(N, 2).contiguous().cuda())
        assert (got.logprobs.cpu().double() + math.log(2.0)).abs().max() <= 2.0 ** -21
        assert (got.entropy.cpu().double() - math.log(2.0)).abs().max() <= 2.0 ** -21


def test_shortlists_of_one_likely_token():
    V, M = 3000, 30
    of = torch.randint(0, M, (V,), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    layout = D.build_layout(of.cuda(), torch.zeros((V, 8), device="cuda"), M)
    sel, off, length, ids = D.shortlist(layout, torch.tensor([[3, 9, 17], [29, 0, 4]], dtype=torch.int32).cuda())
    z = torch.full(ids.shape, float("nan"))
    for r, at in ((0, 11), (1, int(length[1]) - 1)):
        z[r, :int(length[r])] = torch.randn(int(length[r]), generator=torch.Generator().manual_seed(r))
        z[r, at] = 22.0
    names = torch.stack([ids[0, 11], ids[1, int(length[1]) - 1]])
    got = D.token_logprobs(z.cuda(), names, rows=D.ShortlistRows(layout, sel, off, length))
    for r, at in ((0, 11), (1, int(length[1]) - 1)):
        check_row(z[r, :int(length[r])].double().numpy(), 1.0, [float(got.logprobs[r])], float(got.entropy[r]), [at])
