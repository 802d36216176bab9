"""CPU oracle (numpy, fp64) of the target model's side: verification of drafted
chains and trees, distillation from a teacher's top list, the router's loss.

Plain loops over requests and rows from the definitions; shares no code with the
HIP path.  Inputs are fp64 arrays holding the exact values of the device's fp32
or bf16 ones; temperatures and tail weights are the fp32 values the library gets.
"""
from __future__ import annotations

import numpy as np

F32_MAX = 3.4028234663852886e38


def clean(row):
    row = np.where(np.isnan(row), -np.inf, np.asarray(row, dtype=np.float64))
    return np.minimum(row, F32_MAX)


def softmax(row, temperature):
    """Probabilities of a row of logits; all zero where every logit is -inf."""
    z = clean(row)
    m = z.max(initial=-np.inf)
    if m == -np.inf:
        return np.zeros_like(z)
    w = np.exp((z - m) / temperature)
    return w / w.sum()


def place(weights, u):
    """Inverse CDF: the first index whose cumulative weight exceeds u of the total,
    else the last with any weight; -1 without weight."""
    total = weights.sum()
    if not total > 0.0:
        return -1
    F = np.cumsum(weights)
    over = np.nonzero(F > u * F[-1])[0]
    return int(over[0]) if over.size else int(np.nonzero(weights)[0][-1])


def best(row):
    z = clean(row)
    return -1 if z.max(initial=-np.inf) == -np.inf else int(np.argmax(z))


def log_p(row, temperature, x):
    with np.errstate(divide="ignore"):
        return -np.inf if x < 0 else float(np.log(softmax(row, temperature or 1.0)[x]))


def draft_distribution(V, logits, temperature, ids=None, tail=0.0):
    """q over the vocabulary: softmax of the row's logits over `ids` (the shortlist
    in slot order; None: ids 0..len-1), the tail weight spread over the others."""
    ids = np.arange(len(logits)) if ids is None else np.asarray(ids)
    q = np.zeros(V)
    beta = tail if len(ids) < V else 0.0
    q[ids] = (1.0 - beta) * softmax(logits[:len(ids)], temperature)
    if beta > 0.0:
        away = np.ones(V, dtype=bool)
        away[ids] = False
        q[away] = beta / away.sum()
    return q


def verify_chain(target, tokens, uniforms, length, temperature, q_of=None, q_token=None):
    """One request.  target [n + 1, V], tokens [n], uniforms [n + 1]; q_of(i): the
    whole draft distribution of draft i or None (outright), q_token[i] its value
    at the token as the drafter reported it.  -> (accepted, ids, logprobs)."""
    n, V = len(tokens), target.shape[1]
    ids, lps = [], []
    for i in range(n + 1):
        row = target[i]
        x = int(tokens[i]) if i < min(max(length, 0), n) else -1
        if not 0 <= x < V:
            x = -1
        if temperature == 0.0:
            g = best(row)
            ids.append(g)
            lps.append(log_p(row, 1.0, g))
            if x >= 0 and x == g:
                continue
            return i, ids, lps
        p = softmax(row, temperature)
        q = None if x < 0 or q_of is None else q_of(i)
        if x >= 0:
            qx = 1.0 if q is None else float(q_token[i])
            if float(uniforms[i]) * qx < p[x]:
                ids.append(x)
                lps.append(log_p(row, temperature, x))
                continue
        r = p
        if x >= 0:
            r = np.maximum(p - q, 0.0) if q is not None else np.where(np.arange(V) == x, 0.0, p)
            r = r if r.sum() > 0.0 else p
        ids.append(place(r, float(uniforms[n])))
        lps.append(log_p(row, temperature, ids[-1]))
        return i, ids, lps
    raise AssertionError


def verify_tree(target, tokens, parents, uniforms, temperature):
    """One request.  target [N, V].  -> (accepted, ids, logprobs, nodes)."""
    N, V = target.shape
    here, ids, lps, nodes = 0, [], [], []
    while True:
        row = target[here]
        kids = [j for j in range(1, N) if parents[j] == here and here < j and 0 <= tokens[j] < V]
        took = None
        if temperature == 0.0:
            end = best(row)
            took = next((j for j in kids if tokens[j] == end), None)
        else:
            p = softmax(row, temperature)
            r, mass = p.copy(), 1.0
            for j in kids:
                px = r[tokens[j]]
                if float(uniforms[j]) * mass < px:
                    took = j
                    break
                mass -= px
                r[tokens[j]] = 0.0
            if took is None:
                end = place(r if r.sum() > 0.0 else p, float(uniforms[0]))
        ids.append(end if took is None else int(tokens[took]))
        lps.append(log_p(row, temperature, ids[-1]))
        if took is None:
            return len(nodes), ids, lps, nodes
        nodes.append(took)
        here = took


def teacher_entries(ids, V):
    """Indices of a list's entries: ids inside the vocabulary, the first of equal ones."""
    seen, keep = set(), []
    for k, i in enumerate(ids):
        if 0 <= i < V and int(i) not in seen:
            seen.add(int(i))
            keep.append(k)
    return keep


def distill_row(z, ids, values, temperature, tail):
    """Loss, d loss / d z, and (log sum exp over all, over those outside the list)
    of one row of student logits, with the pieces the error bounds need."""
    z = np.asarray(z, dtype=np.float64)
    V = z.size
    keep = teacher_entries(ids, V)
    at = np.asarray([ids[k] for k in keep], dtype=np.int64)
    t = np.asarray([values[k] for k in keep], dtype=np.float64)
    with np.errstate(all="ignore"):
        s = z / temperature
        m = s.max()
        outside = np.ones(V, dtype=bool)
        outside[at] = False
        # sums relative to the largest logit: next to the type's lowest value a
        # log of sums has no digits left for them
        log_q, log_rest, q = np.full(V, -np.inf), -np.inf, np.zeros(V)
        lse = lse_out = -np.inf
        spread_q = np.zeros(V)  # q over q_rest outside the list
        if m > -np.inf:
            total = np.exp(s - m).sum()
            lse, log_q = m + np.log(total), (s - m) - np.log(total)
            q = np.exp(s - m) / total
            so = s[outside]
            mo = so.max(initial=-np.inf)
            if mo > -np.inf:
                part = np.exp(so - mo).sum()
                lse_out, log_rest = mo + np.log(part), (mo - m) + np.log(part) - np.log(total)
                spread_q[outside] = np.exp(so - mo) / part
        if tail:
            lp = t
            rest = max(0.0, 1.0 - np.exp(t).sum()) if len(at) < V else 0.0
        else:
            rest = 0.0
            top = t.max(initial=-np.inf)
            if top == -np.inf:
                return 0.0, np.zeros(V), (lse, lse_out), np.zeros(V)
            lp = (t - top) / temperature
            lp = lp - np.log(np.exp(lp).sum())
        p = np.exp(lp)
        loss = sum(pk * (lk - log_q[i]) for pk, lk, i in zip(p, lp, at) if pk > 0.0)
        if rest > 0.0:
            loss += rest * (np.log(rest) - log_rest)
        if m == -np.inf:
            loss = np.inf
        mass = p.sum() + rest
        grad = mass * q
        size = mass * q
        if rest > 0.0:
            grad = grad - rest * spread_q
            size = size + rest * spread_q
        grad[at] -= p
        size[at] += p
    return loss, grad / temperature, (lse, lse_out), size / temperature


def router_row(s, labels, pos_weight):
    """Loss and gradient of one row of scores, labels a bool array."""
    s = np.asarray(s, dtype=np.float64)
    with np.errstate(all="ignore"):
        x = np.where(labels, -s, s)
        k = np.where(labels, pos_weight, 1.0)
        cost = k * np.logaddexp(0.0, x)
        sig = 1.0 / (1.0 + np.exp(-x))
    return cost, np.where(labels, -k * sig, sig)
