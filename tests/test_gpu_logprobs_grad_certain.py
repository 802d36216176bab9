"""The gradient at a token that has almost all of its row's weight: g (1 - p) - ..., held to a share of 1 - p and not of g.

Statistics come in 64 bits from the definition, so that what is seen is the gradient's own arithmetic; elements of
listed tokens are computed in 64 bits, multiplied by 1 / T rounded, and rounded: 4 steps of 2^-24 and the type's half.
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


def rows(V, dtype, seed, gaps=(0.0, 1.0, 3.0, 5.0, 6.0, 7.5, 9.0, 14.0)):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((len(gaps), V), generator=g) * 0.75
    at = torch.randint(0, V, (len(gaps),), generator=g)
    for r, gap in enumerate(gaps):
        z[r, at[r]] = math.log(V * 10.0 ** gap) + 1.0
    return z.to(DT[dtype]), at


def exact(z, T):
    """(log-probabilities, 1 - p, largest, log s, entropy) of a row whose largest logit stands alone."""
    best = int(z.argmax())
    y = (z - z[best]) / T
    w = np.exp(y)
    w[best] = 0.0
    rest = float(w.sum())
    s = 1.0 + rest
    p = w / s
    p[best] = 1.0 / s
    off = 1.0 - p
    off[best] = rest / s
    H = math.log1p(rest) - float((w * y).sum()) / s
    return y - math.log1p(rest), p, off, z[best], math.log1p(rest), H


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,temperature", [(40, 1.0), (3000, 0.7), (40000, 1.0), (128256, 2.0)])
@pytest.mark.parametrize("entropy", [False, True])
def test_elements_of_likely_tokens(V, temperature, entropy, dtype):
    T = float(np.float32(temperature))
    z, at = rows(V, dtype, V)
    N = z.shape[0]
    gen = torch.Generator().manual_seed(7)
    # the likely token, another, the likely one again, one that is not there
    tokens = torch.stack([at, (at + 3) % V, at, torch.full_like(at, -1)], 1).to(torch.int32)
    g = torch.randn((N, 4), generator=gen)
    g[::2, 1] = 0.0  # rows that name the likely token alone
    e = torch.randn(N, generator=gen) if entropy else None
    stats = torch.zeros((N, 3), dtype=torch.float64)
    rows64 = [exact(z[r].double().numpy(), T) for r in range(N)]
    for r, (_, _, _, m, log_s, H) in enumerate(rows64):
        stats[r] = torch.tensor([m, log_s, H], dtype=torch.float64)
    got = D.token_logprobs_grad(z.cuda(), stats.cuda(), tokens.cuda(), g.cuda(), None if e is None else e.cuda(),
                                temperature=T).double().cpu().numpy()
    half = torch.finfo(DT[dtype]).eps / 2
    for r, (logp, p, off, _, _, H) in enumerate(rows64):
        gg = g[r, :3].double().numpy()
        ee = 0.0 if e is None else float(e[r])
        own = {int(tokens[r, 0]): (gg[0] + gg[2], gg[1]), int(tokens[r, 1]): (gg[1], gg[0] + gg[2])}
        for v, (G, R) in own.items():
            want = (G * off[v] - R * p[v] - ee * p[v] * (logp[v] + H)) / T
            size = (abs(G) * off[v] + abs(R) * p[v] + abs(ee) * p[v] * (abs(logp[v]) + H)) / T
            # (R is a sum in 64 bits of 32-bit numbers, and log s is given to 2^-52 of itself)
            tol = 4 * EPS * size + half * (abs(want) + 4 * EPS * size)
            assert abs(got[r, v] - want) <= tol, (r, v, got[r, v], want, off[v])


@pytest.mark.parametrize("N", [8, 1040])
def test_training_on_certain_rows_goes_to_zero_together(N):
    """Forward and backward calls as a loop makes them: the likely token's element is what the others' lose."""
    V = 20000
    z, at = rows(V, "f32", 3, gaps=(2.0, 3.0, 4.0, 5.0, 6.0, 7.0, 8.0, 9.0))
    z, at = z.repeat(N // 8, 1).cuda(), at.repeat(N // 8).to(torch.int32).cuda()
    s = D.token_logprobs(z, at, want_stats=True)
    g = torch.ones(N, device="cuda")
    grad = D.token_logprobs_grad(z, s.stats, at, g).double().cpu()
    for r in range(8):
        own = float(grad[r, int(at[r])])
        others = float(grad[r].sum()) - own
        _, p, off, _, _, _ = exact(z[r].double().cpu().numpy(), 1.0)
        best = int(at[r])
        # both are r / (1 + r): the forward's share of r (weights 4 |y| 2^-24 + 2^-22 with |y| < 60, sums 2^-21, three
        # sweeps' 2^-22) and the gradient's own roundings (its weights (6 |log p| + 16) 2^-24 with |log p| < 45)
        forward = 4 * 60 * EPS + 2.0 ** -22 + 2.0 ** -21 + 3 * 2.0 ** -22
        assert abs(own - off[best]) <= (forward + 8 * EPS) * off[best], (own, off[best])
        assert abs(others + off[best]) <= (forward + 286 * EPS) * off[best]


def test_a_token_named_many_times_and_by_opposite_signs():
    """Own terms and those of other tokens are summed apart: opposite ones leave what the others ask for."""
    z, at = rows(500, "f32", 5, gaps=(6.0, 8.0))
    tokens = torch.stack([at] * 6 + [(at + 1) % 500], 1).to(torch.int32)
    g = torch.tensor([[1.0, -1.0, 0.5, -0.5, 3.0, -3.0, 0.125]] * 2)
    stats = torch.zeros((2, 3), dtype=torch.float64)
    rows64 = [exact(z[r].double().numpy(), 1.0) for r in range(2)]
    for r, (_, _, _, m, log_s, H) in enumerate(rows64):
        stats[r] = torch.tensor([m, log_s, H], dtype=torch.float64)
    got = D.token_logprobs_grad(z.cuda(), stats.cuda(), tokens.cuda(), g.cuda()).double().cpu()
    for r, (_, p, off, _, _, _) in enumerate(rows64):
        v, other = int(at[r]), int(tokens[r, 6])
        assert abs(float(got[r, v]) + 0.125 * p[v]) <= 6 * EPS * 0.125
        assert abs(float(got[r, other]) - 0.125 * off[other]) <= 6 * EPS * 0.125
