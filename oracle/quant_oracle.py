"""Plain fp64 oracle of the four-bit rows and of the log-probabilities of given tokens (test infrastructure).

Every function follows its definition, row by row, in float64 numpy from the exact input values, and shares no code
with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- four-bit rows
def quantized_value(x: float, scale: float) -> float:
    """The value that x becomes under a scale: the nearest of VALUES (with x's sign) over it, ties to the even
    place in VALUES, the largest one beyond."""
    a = abs(x) / scale
    best = min(range(8), key=lambda i: (abs(a - VALUES[i]), i % 2))
    return math.copysign(VALUES[best] * scale, x)


def block_scale(block) -> float:
    """2^(floor(log2 of the largest magnitude) - 2), at least 2^-127."""
    a = max(abs(float(v)) for v in block)
    if a == 0.0:
        return 2.0 ** -127
    return 2.0 ** max(math.frexp(a)[1] - 1 - 2, -127)


def quantized_rows(x) -> np.ndarray:
    """The values that rows x [rows, d] stand for in four bits, in float64."""
    x = np.asarray(x, dtype=np.float64)
    out = np.empty_like(x)
    for r in range(x.shape[0]):
        for k in range(0, x.shape[1], BLOCK):
            block = x[r, k:k + BLOCK]
            if not np.isfinite(block).all():
                out[r, k:k + BLOCK] = np.nan
                continue
            scale = block_scale(block)
            out[r, k:k + BLOCK] = [quantized_value(float(v), scale) for v in block]
    return out


def product(a, W) -> np.ndarray:
    """Contexts a [B, d] times rows W [n, d] -> [B, n]."""
    return np.asarray(a, dtype=np.float64) @ np.asarray(W, dtype=np.float64).T


def product_sizes(a, W) -> np.ndarray:
    """Sum of the magnitudes of every product's terms, what rounding errors are measured by."""
    return np.abs(np.asarray(a, dtype=np.float64)) @ np.abs(np.asarray(W, dtype=np.float64)).T


# ---------------------------------------------------------------- log-probabilities
def token_logprobs(z, names, tokens, temperature=1.0, top=0):
    """One row: logits z of the tokens `names` -> (log-probabilities of `tokens`, entropy, [(id, log-probability)] of
    the `top` best, log-probabilities of every column)."""
    z = np.asarray(z, dtype=np.float64)
    names = [int(n) for n in names]
    if np.isnan(z).any() or (z == np.inf).any():
        logp = np.full(z.shape, np.nan)
        entropy = float("nan")
    elif z.size == 0 or (z == -np.inf).all():
        logp = np.full(z.shape, -np.inf)
        entropy = 0.0
    else:
        y = (z - z.max()) / temperature
        logp = y - math.log(float(np.exp(y).sum()))
        entropy = float(-sum(math.exp(v) * v for v in logp if v > -np.inf))
    at = {n: i for i, n in enumerate(names)}
    given = [float(logp[at[int(t)]]) if int(t) in at else -np.inf for t in tokens]
    order = sorted((i for i in range(len(names)) if z[i] > -np.inf), key=lambda i: (-z[i], names[i]))
    best = [(names[i], float(logp[i])) for i in order[:top]]
    best += [(-1, -np.inf)] * (top - len(best))
    return np.array(given), entropy, best, logp


def token_logprobs_grad(z, names, tokens, g, e, temperature=1.0):
    """One row's gradient of sum(g * log-probabilities) + e * entropy with respect to z."""
    _, entropy, _, logp = token_logprobs(z, names, tokens, temperature)
    at = {int(n): i for i, n in enumerate(names)}
    out = np.zeros(len(logp))
    used = [(at[int(t)], float(w)) for t, w in zip(tokens, g) if int(t) in at]
    if (all(w == 0.0 for _, w in used) and e == 0.0) or len(logp) == 0 or (logp == -np.inf).all():
        return out
    p = np.exp(logp)
    for i, w in used:
        out -= w * p
        out[i] += w
    if e != 0.0:
        with np.errstate(invalid="ignore"):
            out -= e * np.where(p == 0.0, 0.0, p * (logp + entropy))
    return out / temperature
