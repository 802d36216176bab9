"""Verification of drafted chains and trees against the fp64 oracle.

Ids, lengths and nodes must be equal.  A draft's test compares u q with a p
whose relative error is bounded below, so an input within that bound of the
border could go either way: none of the fixed inputs lies there.  The drawn
token is computed in 64 bits on both sides.

Log-probabilities.  A row's sum of exponentials carries, per term of weight
e^-x, the rounding of x log2(e) (two roundings: 2 * 1.45 x * 2^-24) and of the
exponential (2^-23), and the fp32 sum of eight terms (7 * 2^-24); the mean of x
under the softmax is at most ln V, so log p of a draft that stands is within
(2.9 ln V + 16) 2^-24, and every log-probability is rounded to fp32 once.
"""
import math

import numpy as np
import pytest
import torch

from oracle import target_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    global D
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2510_13847_amd import dynahead
    D = dynahead
    D.lib()
    yield


def f64(t):
    return t.detach().cpu().double().numpy()


def lp_bound(V, lp):
    return (2.9 * math.log(max(V, 2)) + 16) * 2.0 ** -24 + abs(lp) * 2.0 ** -24 + 1e-30


def check(v, b, want, V, nodes=False):
    """Row b of a verifier's outputs against the oracle's (accepted, ids, logprobs[, nodes])."""
    n, ids, lps = want[:3]
    width = v.ids.shape[1]
    assert int(v.lengths[b]) == n, (b, int(v.lengths[b]), n)
    assert v.ids[b].tolist() == ids + [-1] * (width - len(ids)), (b, v.ids[b].tolist(), ids)
    got = v.logprobs[b].tolist()
    for i, (g, w) in enumerate(zip(got, lps)):
        assert g == w or abs(g - w) <= lp_bound(V, w), (b, i, g, w)
    assert all(g == -math.inf for g in got[len(ids):])
    if nodes:
        assert v.nodes[b].tolist() == want[3] + [-1] * (width - len(want[3]))


def layout_of(V, M, seed):
    rng = np.random.default_rng(seed)
    of = rng.integers(0, M, V).astype(np.int32)
    of[rng.permutation(V)[:M]] = np.arange(M)  # no cluster empty
    W = torch.zeros((V, 8), dtype=torch.bfloat16, device=DEV)
    return of, D.build_layout(torch.from_numpy(of).to(DEV), W, M)


def shortlist(of, clusters):
    return np.concatenate([np.nonzero(of == m)[0] for m in sorted(set(clusters))])


def make_steps(B, n, V, kind, seed, M=0, k=0, td=1.0, tail=0.0, target=None):
    """n drafted positions of B chains, sampled from a draft that follows the
    target with an error.  -> (of, layout, steps, q_of(b) -> callable, q_token)."""
    rng = np.random.default_rng(seed)
    td = float(np.float32(td))
    tail = float(np.float32(tail))
    of, layout = layout_of(V, M, seed) if kind in ("clusters", "shared") else (None, None)
    steps, dists = [], []
    for i in range(n):
        z = 0.8 * np.nan_to_num(target[:, i], neginf=-30.0, posinf=30.0) + rng.standard_normal((B, V))
        if kind == "outright":
            tok = z.argmax(1).astype(np.int32)
            steps.append(D.DraftStep(torch.from_numpy(tok).to(DEV)))
            dists.append([None] * B)
            continue
        if kind == "dense":
            ids = [None] * B
            logits = z[:, :max(1, V - V // 3)].astype(np.float32)
            clusters = None
        else:
            clusters = np.stack([rng.permutation(M)[:k] for _ in range(B)]).astype(np.int32)
            shared = kind == "shared" and B > 1
            ids = [shortlist(of, clusters.reshape(-1) if shared else clusters[b]) for b in range(B)]
            cap = D.union_cap(layout, B, k) if shared else layout.cap(k)
            logits = np.full((B, cap), np.nan, dtype=np.float32)
            for b in range(B):
                logits[b, :len(ids[b])] = z[b, ids[b]]
        row = [O.draft_distribution(V, logits[b].astype(np.float64), td, ids[b], tail) for b in range(B)]
        tok = np.array([O.place(q, rng.random()) for q in row], dtype=np.int32)
        lp = np.array([np.log(row[b][tok[b]]) for b in range(B)], dtype=np.float32)
        steps.append(D.DraftStep(torch.from_numpy(tok).to(DEV), torch.from_numpy(lp).to(DEV),
                                 torch.from_numpy(logits).to(DEV),
                                 None if clusters is None else torch.from_numpy(clusters).to(DEV), td, tail,
                                 kind == "shared" and B > 1))
        dists.append(row)
    return of, layout, steps, dists


def chain_oracle(target, steps, dists, u, lens, T, b):
    n = len(steps)
    tokens = [int(s.tokens[b]) for s in steps]
    qt = [math.exp(float(s.logprobs[b])) if s.logprobs is not None else 1.0 for s in steps]
    return O.verify_chain(target[b], tokens, u[b], n if lens is None else int(lens[b]), T,
                          lambda i: dists[i][b], qt)


CHAINS = [  # V, B, n, dtype, T, kind, kwargs
    (1, 2, 1, "f32", 1.0, "outright", {}),
    (1, 1, 2, "bf16", 0.0, "outright", {}),
    (5, 3, 2, "f32", 1.0, "dense", {}),
    (7, 4, 0, "bf16", 1.0, "outright", {}),
    (2047, 3, 5, "bf16", 1.0, "clusters", dict(M=16, k=4)),
    (2048, 2, 3, "f32", 0.7, "clusters", dict(M=8, k=8, td=0.9)),           # k = M: an empty complement
    (2049, 5, 4, "bf16", 1.3, "clusters", dict(M=40, k=3, tail=0.1, td=0.8)),
    (8191, 4, 3, "f32", 1.0, "shared", dict(M=32, k=3)),
    (8191, 1, 3, "bf16", 1.0, "shared", dict(M=32, k=3, tail=0.25)),
    (4099, 6, 6, "bf16", 0.0, "clusters", dict(M=16, k=4)),
    (50021, 3, 5, "bf16", 1.0, "clusters", dict(M=300, k=24)),
    (50021, 2, 32, "bf16", 1.0, "outright", {}),
    (131077, 2, 4, "f32", 0.6, "dense", dict(td=1.1)),
    (100003, 2, 2, "bf16", 1.0, "clusters", dict(M=40, k=25)),              # a shortlist longer than 32768
    (20011, 2, 2, "f32", 1.0, "clusters", dict(M=2500, k=2100)),            # more clusters than a list in LDS holds
]


@pytest.mark.parametrize("V,B,n,dtype,T,kind,kw", CHAINS)
@pytest.mark.parametrize("ragged", [False, True])
def test_chain(V, B, n, dtype, T, kind, kw, ragged):
    T = float(np.float32(T))
    seed = V + 17 * B + n + ragged
    rng = np.random.default_rng(seed)
    t = torch.from_numpy(3.0 * rng.standard_normal((B, n + 1, V)).astype(np.float32))
    t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    target = f64(t)
    of, layout, steps, dists = make_steps(B, n, V, kind, seed + 1, target=target, **kw)
    u = rng.random((B, n + 1)).astype(np.float32)
    u[rng.random((B, n + 1)) < 0.4] *= 0.05  # more drafts stand
    lens = rng.integers(0, n + 2, B).astype(np.int32) if ragged else None
    if ragged and n > 1:
        steps[n // 2].tokens[0] = -1  # no token proposed: the chain ends there
        lens[B - 1] = -3
    v = D.verify_chain(t.to(DEV), steps, torch.from_numpy(u).to(DEV),
                       None if lens is None else torch.from_numpy(lens).to(DEV), T, layout)
    for b in range(B):
        check(v, b, chain_oracle(target, steps, dists, u, None if lens is None else np.clip(lens, 0, n), T, b), V)


@pytest.mark.parametrize("V,B,n,kind,kw", [
    (7, 5000, 1, "outright", {}), (11, 3000, 2, "clusters", dict(M=4, k=2, tail=0.2)), (40, 2000, 3, "shared", dict(M=9, k=1)),
    (2049, 700, 2, "dense", {}), (3001, 600, 1, "clusters", dict(M=200, k=20))])
def test_chain_many_requests(V, B, n, kind, kw):
    """More requests than the chip holds workgroups."""
    rng = np.random.default_rng(V)
    t = torch.from_numpy(2.0 * rng.standard_normal((B, n + 1, V)).astype(np.float32))
    target = f64(t)
    _, layout, steps, dists = make_steps(B, n, V, kind, V + 1, target=target, **kw)
    u = rng.random((B, n + 1)).astype(np.float32)
    v = D.verify_chain(t.to(DEV), steps, torch.from_numpy(u).to(DEV), None, 1.0, layout)
    got = (v.lengths.cpu(), v.ids.cpu(), v.logprobs.cpu())
    fields = [(s.tokens.cpu(), s.logprobs.cpu() if s.logprobs is not None else None) for s in steps]
    rows = range(B) if B * V < 200000 else rng.integers(0, B, 60)
    for b in rows:
        q = [math.exp(float(lp[b])) if lp is not None else 1.0 for _, lp in fields]
        want = O.verify_chain(target[b], [int(x[b]) for x, _ in fields], u[b], n, 1.0, lambda i: dists[i][b], q)
        ids = got[1][b].tolist()
        assert (int(got[0][b]), ids) == (want[0], want[1] + [-1] * (n + 1 - len(want[1]))), b
        for g, w in zip(got[2][b].tolist(), want[2]):
            assert abs(g - w) <= lp_bound(V, w), (b, g, w)


@pytest.mark.parametrize("T", [0.0, 1.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chain_masked_rows(T, dtype):
    """Rows with -inf, NaN, +inf, the type's lowest value, and rows that allow
    nothing, one token, or the drafted token only."""
    V, n = 4100, 2
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    low = torch.finfo(dt).min
    rng = np.random.default_rng(3)
    base = torch.from_numpy(2.0 * rng.standard_normal((10, n + 1, V)).astype(np.float32)).to(dt)
    base[0, 0] = -math.inf                       # nothing allowed
    base[1, 0] = math.nan                        # nothing either
    base[2, 0] = low                             # all equal
    base[3, 0, :-1] = -math.inf                  # the last token only
    base[4, 0, 5:] = low                         # five tokens
    base[5, 0, 77] = math.inf                    # one certain token
    base[6, 0, [3, 4000]] = math.inf             # two of them
    base[7, 0, ::2] = math.nan
    base[8, 0, :] = -math.inf
    base[8, 0, 9] = 1.0                          # the drafted token alone
    base[9, 0, :4000] = -math.inf
    tok = np.full((10, n), 9, dtype=np.int32)
    tok[3] = V - 1
    tok[5] = 77
    tok[6] = 3
    steps = [D.DraftStep(torch.from_numpy(tok[:, i].copy()).to(DEV)) for i in range(n)]
    dists = [[None] * 10] * n
    for us in (0.0, 0.3, 0.999):
        u = np.full((10, n + 1), us, dtype=np.float32)
        v = D.verify_chain(base.to(DEV), steps, torch.from_numpy(u).to(DEV), None, T)
        for b in range(10):
            check(v, b, chain_oracle(f64(base), steps, dists, u, None, T, b), V)
    assert v.ids[0].tolist() == [-1, -1, -1] and v.ids[1].tolist() == [-1, -1, -1]


def test_greedy_ties_go_to_the_lower_id():
    V = 20000
    t = torch.zeros((3, 2, V), dtype=torch.bfloat16)
    t[0, 0, [19999, 4097, 300]] = 2.0
    t[1, 0, 5] = 0.0
    t[1, 0, :5] = -0.0                            # -0 equals +0
    t[2] = -1.0
    t[2, 0, [8000, 12000]] = 7.0
    tok = torch.tensor([300, 5, 12000], dtype=torch.int32, device=DEV)
    v = D.verify_chain(t.to(DEV), [D.DraftStep(tok)], None, None, 0.0)
    assert v.lengths.tolist() == [1, 0, 0]
    assert v.ids.tolist() == [[300, 0], [0, -1], [8000, -1]]


@pytest.mark.parametrize("T", [1.2e-38, 1e-20, 1e20, 2.9e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures_at_their_ends(T, dtype):
    """One-hot and flat targets: all weight on the largest logits, equal ones
    among them, or the same weight on every token."""
    T = float(np.float32(T))
    V, B, n = 2500, 6, 2
    g = torch.Generator().manual_seed(77)
    t = (3.0 * torch.randn((B, n + 1, V), generator=g)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    t[1, :, 40:44] = 20.0
    t[2] = 0.0
    t[3, :, 5] = 100.0
    target = f64(t)
    _, _, steps, dists = make_steps(B, n, V, "outright", 3, target=target)
    u = np.random.default_rng(8).random((B, n + 1)).astype(np.float32)
    v = D.verify_chain(t.to(DEV), steps, torch.from_numpy(u).to(DEV), None, T)
    for b in range(B):
        check(v, b, chain_oracle(target, steps, dists, u, None, T, b), V)


def test_uniforms_at_their_ends():
    """u = 0 accepts any token of some probability and draws the first one; the
    largest u below 1 draws the last one with weight."""
    V = 6000
    t = torch.full((2, 2, V), -math.inf)
    t[:, :, 100:5900] = 0.0
    tok = torch.tensor([50, 5000], dtype=torch.int32, device=DEV)
    for u, want in ((0.0, [[100, -1], [5000, 100]]), (1.0 - 2.0 ** -24, [[5899, -1], [5899, -1]])):
        uu = torch.full((2, 2), u, device=DEV)
        v = D.verify_chain(t.to(DEV), [D.DraftStep(tok)], uu)
        assert v.ids.tolist() == want


def test_residual_without_mass_falls_back_to_the_target():
    """p = q: a draft falls only by its reported probability (here made larger);
    nothing is left of p, and the token is drawn from p."""
    V = 3000
    g = torch.Generator().manual_seed(5)
    z = torch.randn((2, V), generator=g)
    t = torch.stack([z, z], 1)
    tok = torch.tensor([7, 8], dtype=torch.int32, device=DEV)
    step = D.DraftStep(tok, torch.zeros(2, device=DEV), z.to(DEV))
    u = torch.full((2, 2), 0.75, device=DEV)
    v = D.verify_chain(t.to(DEV), [step], u)
    for b in range(2):
        assert int(v.lengths[b]) == 0 and int(v.ids[b, 0]) == O.place(O.softmax(f64(z)[b], 1.0), 0.75)


def test_chain_strided_target_and_untouched_neighbours():
    """Rows inside a larger buffer, at odd element offsets, on a side stream."""
    V, B, n = 5003, 3, 3
    g = torch.Generator().manual_seed(11)
    big = (3.0 * torch.randn((B, n + 3, V + 5), generator=g)).to(torch.bfloat16).to(DEV)
    t = big[:, 1:n + 2, 3:V + 3]
    target = f64(t)
    of, layout, steps, dists = make_steps(B, n, V, "clusters", 2, M=20, k=5, target=target)
    u = np.random.default_rng(1).random((B, n + 1)).astype(np.float32)
    ver = D.ChainVerifier(B, n, V, 1.0, layout)
    uu = torch.from_numpy(u).to(DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ver(t, steps, uu, stream=side)
    side.synchronize()
    for b in range(B):
        check(ver, b, chain_oracle(target, steps, dists, u, None, 1.0, b), V)


def test_chain_on_a_stream_that_did_not_make_the_verifier():
    """The verifier's own table of the layout is whole before a call on another
    stream reads it, whatever stood before it on the stream that made it.  The
    shortlist is too long for one workgroup, so every slot is found in the table."""
    V, B, n = 50021, 2, 2
    g = torch.Generator().manual_seed(31)
    t = (3.0 * torch.randn((B, n + 1, V), generator=g)).to(torch.bfloat16).to(DEV)
    target = f64(t)
    of, layout, steps, dists = make_steps(B, n, V, "clusters", 8, M=20, k=16, target=target)
    assert steps[0].logits.shape[1] > 32768
    u = np.random.default_rng(3).random((B, n + 1)).astype(np.float32)
    u[:, 0] = 0.9999  # most first drafts fall: the residual is drawn
    uu = torch.from_numpy(u).to(DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy = torch.ones((4096, 4096), device=DEV)
    for _ in range(20):
        busy = busy @ busy * 1e-4
    ver = D.ChainVerifier(B, n, V, 1.0, layout)
    ver(t, steps, uu, stream=side)
    fresh = D.verify_chain(t, steps, uu, temperature=1.0, layout=layout, stream=side)
    side.synchronize()
    for b in range(B):
        want = chain_oracle(target, steps, dists, u, None, 1.0, b)
        check(ver, b, want, V)
        check(fresh, b, want, V)


def test_two_verifiers_at_once():
    """Calls on two streams, each with its own verifier, leave each other alone."""
    V, B, n = 32003, 4, 3
    runs = []
    for seed in (5, 6):
        g = torch.Generator().manual_seed(seed)
        t = (3.0 * torch.randn((B, n + 1, V), generator=g)).to(torch.bfloat16).to(DEV)
        target = f64(t)
        _, layout, steps, dists = make_steps(B, n, V, "clusters", seed, M=64, k=9, target=target)
        u = np.random.default_rng(seed).random((B, n + 1)).astype(np.float32)
        runs.append((t, target, steps, dists, u, torch.from_numpy(u).to(DEV), D.ChainVerifier(B, n, V, 1.0, layout),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for t, _, steps, _, _, uu, ver, s in runs:
            ver(t, steps, uu, stream=s)
    torch.cuda.synchronize()
    for t, target, steps, dists, u, _, ver, _ in runs:
        for b in range(B):
            check(ver, b, chain_oracle(target, steps, dists, u, None, 1.0, b), V)


def test_chain_rows_beyond_32_bit_offsets():
    V, n = 3001, 1
    stride = (1 << 32) // 2 + 1001               # elements: the second request starts past 4 GiB
    buf = torch.zeros(stride + (n + 1) * V, dtype=torch.bfloat16, device=DEV)
    t = torch.as_strided(buf, (2, n + 1, V), (stride, V, 1))
    g = torch.Generator().manual_seed(4)
    t.copy_((3.0 * torch.randn((2, n + 1, V), generator=g)).to(torch.bfloat16))
    target = f64(t)
    _, layout, steps, dists = make_steps(2, n, V, "outright", 6, target=target)
    u = np.full((2, n + 1), 0.9, dtype=np.float32)
    v = D.verify_chain(t, steps, torch.from_numpy(u).to(DEV))
    for b in range(2):
        check(v, b, chain_oracle(target, steps, dists, u, None, 1.0, b), V)


def test_clusters_out_of_range_or_repeated_are_ignored():
    V, M, k = 4000, 25, 4
    rng = np.random.default_rng(8)
    t = torch.from_numpy(3.0 * rng.standard_normal((1, 2, V)).astype(np.float32))
    of, layout = layout_of(V, M, 8)
    for raw in ([3, 3, 9, 1], [-1, 30, 9, 2], [-1, -1, -1, 99]):
        ids = [m for m in sorted(set(raw)) if 0 <= m < M]
        slots = np.concatenate([np.nonzero(of == m)[0] for m in ids]) if ids else np.empty(0, dtype=np.int64)
        logits = np.full((1, layout.cap(k)), 50.0, dtype=np.float32)
        logits[0, :len(slots)] = rng.standard_normal(len(slots))
        q = O.draft_distribution(V, logits[0].astype(np.float64), 1.0, slots) if ids else np.zeros(V)
        step = D.DraftStep(torch.tensor([11], dtype=torch.int32, device=DEV), torch.zeros(1, device=DEV),
                           torch.from_numpy(logits).to(DEV), torch.tensor([raw], dtype=torch.int32, device=DEV))
        u = torch.tensor([[0.999, 0.6]], device=DEV)
        v = D.verify_chain(t.to(DEV), [step], u, None, 1.0, layout)
        want = O.verify_chain(f64(t)[0], [11], f64(u)[0], 1, 1.0, lambda i: q, [1.0])
        check(v, 0, want, V)


@pytest.mark.parametrize("V,dtype", [(130003, torch.bfloat16), (65003, torch.float32)])
def test_greedy_walks_that_end_in_leaves(V, dtype):
    """Large greedy calls read a leaf's row only where a walk ends in it: rows of
    all kinds behind such walks, masked ones and ones of equal logits among them."""
    B, N = 28, 30
    g = torch.Generator().manual_seed(2)
    t = torch.empty((B, N, V)).normal_(0.0, 3.0, generator=g).to(dtype)
    parents = torch.tensor([0] + [(j - 1) // 2 for j in range(1, N)], dtype=torch.int32)
    tokens = torch.full((B, N), 3, dtype=torch.int32)
    for b in range(B):
        for j in range(1, N):
            if (j + b) % 2 or b in (3, 4, 5):  # the parent's best token
                tokens[b, j] = int(t[b, (j - 1) // 2].float().argmax())
    t[3, 15:] = -math.inf
    t[4, 15:] = 1.0
    t[5, 15:] = math.nan
    v = D.verify_tree(t.to(DEV), tokens.to(DEV), parents.to(DEV), None, 0.0)
    leaves = set()
    for b in range(B):
        want = O.verify_tree(f64(t[b]), tokens[b].tolist(), parents.tolist(), [0.0] * N, 0.0)
        check(v, b, want, V, nodes=True)
        if want[0] == 4:
            leaves.add(b)
    assert {3, 4, 5} <= leaves and len(leaves) >= 5


def random_tree(N, rng, spread):
    parents = np.zeros(N, dtype=np.int32)
    for j in range(1, N):
        parents[j] = rng.integers(max(0, j - spread), j)
    return parents


TREES = [  # V, B, N, dtype, T
    (1, 1, 1, "f32", 1.0), (1, 2, 3, "bf16", 0.0), (9, 5, 12, "f32", 1.0), (2049, 3, 27, "bf16", 0.8),
    (2049, 3, 27, "bf16", 0.0), (300, 2, 1024, "f32", 1.0), (8191, 4, 64, "f32", 1.0), (50021, 2, 65, "bf16", 1.0),
    (128256, 1, 61, "bf16", 1.0),
]


@pytest.mark.parametrize("V,B,N,dtype,T", TREES)
@pytest.mark.parametrize("static", [True, False])
def test_tree(V, B, N, dtype, T, static):
    T = float(np.float32(T))
    rng = np.random.default_rng(V + N + B)
    t = torch.from_numpy(3.0 * rng.standard_normal((B, N, V)).astype(np.float32))
    t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    target = f64(t)
    parents = np.stack([random_tree(N, rng, 10)] * B if static else [random_tree(N, rng, 10) for _ in range(B)])
    tokens = np.zeros((B, N), dtype=np.int32)
    for b in range(B):
        for j in range(1, N):  # among the parent's likely tokens, equal siblings included
            order = np.argsort(-target[b, parents[b, j]])
            tokens[b, j] = order[min(V - 1, rng.integers(0, 6))]
    if N > 8:  # absent nodes
        tokens[:, 5] = -1
        tokens[:, 6] = V
        if not static:
            parents[:, 7] = 7
            parents[:, 8] = -2
    u = rng.random((B, N)).astype(np.float32)
    u[:, 1:][rng.random((B, N - 1)) < 0.3] *= 0.1
    v = D.verify_tree(t.to(DEV), torch.from_numpy(tokens).to(DEV),
                      torch.from_numpy(parents[0] if static else parents).to(DEV), torch.from_numpy(u).to(DEV), T)
    for b in range(B):
        check(v, b, O.verify_tree(target[b], tokens[b], parents[b], u[b], T), V, nodes=True)


@pytest.mark.parametrize("kind", ["chain", "tree", "outright"])
def test_emitted_tokens_are_distributed_as_the_target(kind):
    """The first emitted token of many requests with one target row and fresh
    uniforms: counts within five standard deviations of p."""
    V, B = 12, 40000
    rng = np.random.default_rng(9)
    row = torch.from_numpy(1.2 * rng.standard_normal((1, 1, V)).astype(np.float32))
    p = O.softmax(f64(row)[0, 0], 1.0)
    if kind == "tree":
        t = row.expand(B, 4, V).contiguous().to(DEV)
        tokens = torch.tensor([[0, 3, 5, 2]], dtype=torch.int32).expand(B, 4).contiguous().to(DEV)
        u = torch.from_numpy(rng.random((B, 4)).astype(np.float32)).to(DEV)
        v = D.verify_tree(t, tokens, torch.zeros(4, dtype=torch.int32, device=DEV), u)
    else:
        t = row.expand(B, 2, V).contiguous().to(DEV)
        u = torch.from_numpy(rng.random((B, 2)).astype(np.float32)).to(DEV)
        if kind == "outright":
            step = D.DraftStep(torch.full((B,), 4, dtype=torch.int32, device=DEV))
        else:
            z = rng.standard_normal(9).astype(np.float32)
            q = O.draft_distribution(V, z.astype(np.float64), 1.0)
            tok = rng.choice(V, size=B, p=q).astype(np.int32)
            step = D.DraftStep(torch.from_numpy(tok).to(DEV),
                               torch.from_numpy(np.log(q[tok]).astype(np.float32)).to(DEV),
                               torch.from_numpy(np.broadcast_to(z, (B, 9)).copy()).to(DEV))
        v = D.verify_chain(t, [step], u)
    counts = np.bincount(v.ids[:, 0].cpu().numpy(), minlength=V)
    assert (np.abs(counts - B * p) <= 5.0 * np.sqrt(B * p * (1 - p)) + 1).all(), (counts, B * p)


def test_repeat_runs_and_captured_graphs_agree():
    """Bit-identical results from run to run; a graph replayed several times with
    eager work of another verifier between gives the eager result on new inputs."""
    V, B, n = 9001, 4, 3
    rng = np.random.default_rng(21)

    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        return (3.0 * torch.randn((B, n + 1, V), generator=g)).to(torch.bfloat16).to(DEV), \
            torch.rand((B, n + 1), generator=g).to(DEV)
    t, u = inputs(1)
    _, layout, steps, _ = make_steps(B, n, V, "clusters", 3, M=30, k=6, target=f64(t))
    tree_u = torch.rand((B, n + 1), device=DEV)
    parents = torch.tensor([0, 0, 1, 1], dtype=torch.int32, device=DEV)
    tokens = torch.randint(0, V, (B, n + 1), dtype=torch.int32, device=DEV)
    a, e = (D.ChainVerifier(B, n, V, 1.0, layout) for _ in range(2))
    tr, te = (D.TreeVerifier(B, n + 1, V, 1.0) for _ in range(2))
    for _ in range(2):
        a(t, steps, u)
        tr(t, tokens, parents, tree_u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a(t, steps, u)
        tr(t, tokens, parents, tree_u)
    for seed in range(5):
        nt, nu = inputs(10 + seed)
        t.copy_(nt)
        u.copy_(nu)
        tree_u.copy_(nu)
        e(t, steps, u)
        te(t, tokens, parents, tree_u)
        first = [x.clone() for x in (e.lengths, e.ids, e.logprobs, te.ids, te.nodes, te.logprobs)]
        graph.replay()
        e(t, steps, u)
        torch.cuda.synchronize()
        for x, y in zip(first, (a.lengths, a.ids, a.logprobs, tr.ids, tr.nodes, tr.logprobs)):
            assert torch.equal(x, y)
        assert torch.equal(first[1], e.ids) and torch.equal(first[2], e.logprobs)


def test_verifier_refuses_what_does_not_fit():
    V, B, n = 100, 2, 2
    ver = D.ChainVerifier(B, n, V)
    t = torch.zeros((B, n + 1, V), device=DEV)
    u = torch.zeros((B, n + 1), device=DEV)
    s = D.DraftStep(torch.zeros(B, dtype=torch.int32, device=DEV))
    for bad in (lambda: ver(t[:, :2], [s, s], u), lambda: ver(t, [s], u), lambda: ver(t, [s, s]),
                lambda: ver(t, [s, s], u[:, :2]), lambda: ver(t.transpose(1, 2), [s, s], u),
                lambda: ver(t.cpu(), [s, s], u),
                lambda: D.DraftStep(s.tokens, None, t[:, 0].contiguous()),
                lambda: ver(t, [s, s], u, torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ver(t.half(), [s, s], u)
    with pytest.raises(TypeError):
        D.DraftStep(s.tokens.long())
    with pytest.raises(D.DynaError) as err:
        D.ChainVerifier(B, 33, V)(torch.zeros((B, 34, V), device=DEV), [s] * 33, torch.zeros((B, 34), device=DEV))
    assert err.value.status == D.ERR_UNSUPPORTED
    of, layout = layout_of(V, 10, 1)
    short = D.DraftStep(s.tokens, torch.zeros(B, device=DEV), torch.zeros((B, 1), device=DEV),
                        torch.zeros((B, 3), dtype=torch.int32, device=DEV))
    with pytest.raises(D.DynaError) as err:
        D.verify_chain(t, [short, short], u, None, 1.0, layout)
    assert err.value.status == D.ERR_CAPACITY


def masked_problem(kind, dtype, B, V, M=0, k=0, td=1.0, tail=0.0, allowed=40, seed=0):
    """Rows that allow a few tokens, all of them on the draft's shortlist; the draft
    proposed a token that the target forbids.  -> (target, steps, layout, q of each row)."""
    rng = np.random.default_rng(seed)
    td, tail = float(np.float32(td)), float(np.float32(tail))
    clusters = layout = None
    if kind == "dense":
        ids = [np.arange(V - V // 5)] * B
        cap = V - V // 5
    else:
        of, layout = layout_of(V, M, seed)
        clusters = np.stack([rng.permutation(M)[:k] for _ in range(B)]).astype(np.int32)
        shared = kind == "shared"
        union = shortlist(of, clusters.reshape(-1)) if shared else None
        ids = [union if shared else shortlist(of, c) for c in clusters]
        cap = D.union_cap(layout, B, k) if shared else layout.cap(k)
    target = torch.full((B, 2, V), -math.inf)
    logits = np.full((B, cap), np.nan, dtype=np.float32)
    tokens = np.zeros(B, dtype=np.int32)
    for b in range(B):
        at = rng.permutation(len(ids[b]))[:allowed]
        z = (3.0 * rng.standard_normal(len(at))).astype(np.float32)
        target[b, 0, torch.from_numpy(ids[b][at])] = torch.from_numpy(z)
        # every other draft is masked as the target is
        logits[b, :len(ids[b])] = -np.inf if b % 2 else rng.standard_normal(len(ids[b])) - 4.0
        logits[b, at] = 0.8 * z + rng.standard_normal(len(at))
        tokens[b] = next(v for v in rng.integers(0, V, V) if v not in ids[b][at])
    target[:, 1] = 0.0
    target = target.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q = [O.draft_distribution(V, logits[b].astype(np.float64), td, ids[b], tail) for b in range(B)]
    step = D.DraftStep(torch.from_numpy(tokens).to(DEV), torch.zeros(B, device=DEV), torch.from_numpy(logits).to(DEV),
                       None if clusters is None else torch.from_numpy(clusters).to(DEV), td, tail, kind == "shared")
    return target, step, layout, q, tokens


MASKED = [  # kind, dtype, T, V, kwargs
    ("clusters", "f32", 1.0, 8192, dict(M=16, k=4)), ("clusters", "f32", 1.0, 8192, dict(M=8, k=8)),
    ("clusters", "bf16", 0.75, 8191, dict(M=16, k=4, td=0.9, tail=0.25)),
    ("clusters", "f32", 1.0, 8192, dict(M=8, k=8, tail=0.25)),                       # no token for the tail
    ("shared", "bf16", 1.0, 8192, dict(M=200, k=1)), ("shared", "f32", 1.25, 9001, dict(M=300, k=1, tail=0.125)),
    ("dense", "bf16", 1.0, 8192, {}), ("clusters", "f32", 1.0, 20011, dict(M=2500, k=2100)),
]


@pytest.mark.parametrize("kind,dtype,T,V,kw", MASKED)
@pytest.mark.parametrize("u", [0.0, 2.0 ** -24, 1.0 - 2.0 ** -24])
def test_draws_behind_a_shortlist_hold_to_the_residual(kind, dtype, T, V, kw, u):
    """Whole stretches of the row are emptied by the drafts or masked: the token
    drawn has p > q wherever u points, at its ends too."""
    B = 200
    target, step, layout, q, tokens = masked_problem(kind, dtype, B, V, **kw)
    us = torch.tensor([[0.75, u]]).repeat(B, 1)
    v = D.verify_chain(target.to(DEV), [step], us.to(DEV), None, T, layout)
    for b in range(B):
        row = f64(target[b])
        p = O.softmax(row[0], T)
        some = p > 0
        # sums of 200 terms and of differences are right to 1e-13 of the total: no border is near
        assert (np.abs(p - q[b])[some] > 1e-9 * p[some]).all()
        F = np.cumsum(np.maximum(p - q[b], 0.0))
        assert u == 0.0 or np.abs(F / F[-1] - u).min() > 1e-11
        check(v, b, O.verify_chain(row, [int(tokens[b])], [0.75, u], 1, T, lambda i: q[b], [1.0]), V)
        x = int(v.ids[b, 0])
        assert p[x] > q[b][x] and math.isfinite(float(v.logprobs[b, 0]))


@pytest.mark.parametrize("M,k", [(16, 16), (2500, 2500)])
def test_equal_distributions_over_a_shortlist_leave_the_target(M, k):
    """p = q over a shortlist of the whole vocabulary: nothing is left, whatever u."""
    V = 20000
    of, layout = layout_of(V, M, 4)
    z = torch.randn((4, V), generator=torch.Generator().manual_seed(6)) * 3.0
    ids = torch.from_numpy(shortlist(of, range(M)))
    clusters = torch.arange(M, dtype=torch.int32).repeat(4, 1)
    step = D.DraftStep(torch.full((4,), 9, dtype=torch.int32, device=DEV), torch.zeros(4, device=DEV),
                       z[:, ids].contiguous().to(DEV), clusters.to(DEV))
    t = torch.stack([z, z], 1)
    for u in (0.0, 0.25, 0.75, 1.0 - 2.0 ** -24):
        us = torch.tensor([[0.999, u]]).repeat(4, 1)
        v = D.verify_chain(t.to(DEV), [step], us.to(DEV), None, 1.0, layout)
        for b in range(4):
            assert int(v.lengths[b]) == 0 and int(v.ids[b, 0]) == O.place(O.softmax(f64(z[b]), 1.0), u)


@pytest.mark.parametrize("d,u", [(0.45257025957107544, 0.3887498378753662), (1.6673763990402222, 0.15877428650856018),
                                 (6.1758198738098145, 0.002074786927551031)])
@pytest.mark.parametrize("first,second,V", [(0, 1, 2), (3, 4097, 5000)])
def test_draws_next_to_a_border(d, u, first, second, V):
    """Two tokens d apart, u below p of the first by 3 to 7 parts in 10^14 of it:
    weights in 64 bits draw the first, ones right to 43 bits the second."""
    from decimal import Decimal, getcontext
    getcontext().prec = 40
    w = (-Decimal(d)).exp()
    assert Decimal("2e-14") < (w - Decimal(u) * (1 + w)) / w < Decimal("8e-14")
    t = torch.full((2, 1, V), -math.inf)
    t[:, :, first], t[:, :, second] = -d, 0.0
    us = torch.tensor([[u], [float(np.nextafter(np.float32(u), np.float32(1.0)))]])
    for v in (D.verify_chain(t.to(DEV), [], us.to(DEV)),
              D.verify_tree(t.to(DEV), torch.zeros((2, 1), dtype=torch.int32, device=DEV),
                            torch.zeros(1, dtype=torch.int32, device=DEV), us.to(DEV))):
        assert v.ids.tolist() == [[first], [second]]


LARGEST = [  # V, B, n, dtype, T, kind, kwargs: more chunks than the drawing kernel's threads, up to the limit
    (524801, 2, 2, "bf16", 1.0, "clusters", dict(M=2048, k=10)),
    (1 << 20, 2, 2, "bf16", 1.0, "clusters", dict(M=4096, k=8)),
    (1 << 20, 1, 2, "f32", 0.75, "clusters", dict(M=4096, k=64, tail=0.125)),
    ((1 << 20) - 1, 3, 1, "bf16", 1.0, "shared", dict(M=4096, k=8)),
    (1 << 20, 1, 1, "f32", 1.0, "clusters", dict(M=100, k=5)),              # a shortlist longer than 32768
    (1 << 20, 2, 1, "bf16", 1.0, "dense", {}), (1 << 20, 2, 3, "bf16", 1.0, "outright", {}),
    (1 << 20, 2, 3, "f32", 0.0, "outright", {}),
]


@pytest.mark.parametrize("V,B,n,dtype,T,kind,kw", LARGEST)
def test_chain_over_the_largest_vocabularies(V, B, n, dtype, T, kind, kw):
    rng = np.random.default_rng(V + n)
    t = torch.from_numpy(3.0 * rng.standard_normal((B, n + 1, V), dtype=np.float32))
    t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    target = f64(t)
    _, layout, steps, dists = make_steps(B, n, V, kind, V + 1, target=target, **kw)
    td = t.to(DEV)
    ver = D.ChainVerifier(B, n, V, T, layout)
    for last in (0.0, 0.37, 0.999, 1.0 - 2.0 ** -24):
        u = rng.random((B, n + 1)).astype(np.float32)
        u[:, 0] = 0.999 if last < 0.5 else 0.001  # most first drafts fall, most stand
        u[:, n] = last
        ver(td, steps, torch.from_numpy(u).to(DEV))
        for b in range(B):
            check(ver, b, chain_oracle(target, steps, dists, u, None, T, b), V)


@pytest.mark.parametrize("kind,V,kw", [("clusters", 1 << 20, dict(M=4096, k=8)), ("dense", 600011, {}),
                                       ("clusters", 600011, dict(M=4096, k=8, tail=0.25))])
@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24])
def test_draws_over_the_largest_vocabularies_hold_to_the_residual(kind, V, kw, u):
    B = 12
    target, step, layout, q, tokens = masked_problem(kind, "f32", B, V, allowed=150, **kw)
    us = torch.tensor([[0.75, u]]).repeat(B, 1)
    v = D.verify_chain(target.to(DEV), [step], us.to(DEV), None, 1.0, layout)
    for b in range(B):
        check(v, b, O.verify_chain(f64(target[b]), [int(tokens[b])], [0.75, u], 1, 1.0, lambda i: q[b], [1.0]), V)


@pytest.mark.parametrize("T", [0.0, 1.0])
def test_tree_over_the_largest_vocabulary(T):
    V, B, N = 1 << 20, 2, 6
    rng = np.random.default_rng(12)
    t = torch.from_numpy(3.0 * rng.standard_normal((B, N, V), dtype=np.float32)).to(torch.bfloat16)
    target = f64(t)
    parents = np.array([0, 0, 0, 1, 2, 3], dtype=np.int32)
    tokens = np.zeros((B, N), dtype=np.int32)
    for b in range(B):
        for j in range(1, N):
            tokens[b, j] = np.argsort(-target[b, parents[j]])[rng.integers(0, 2)]
    for last in (0.0, 0.5, 1.0 - 2.0 ** -24):
        u = (rng.random((B, N)) * 0.01).astype(np.float32)
        u[:, 0] = last
        v = D.verify_tree(t.to(DEV), torch.from_numpy(tokens).to(DEV), torch.from_numpy(parents).to(DEV),
                          torch.from_numpy(u).to(DEV), T)
        for b in range(B):
            check(v, b, O.verify_tree(target[b], tokens[b], parents, u[b], T), V, nodes=True)


@pytest.mark.parametrize("kind,V,kw", [("clusters", 50021, dict(M=64, k=8)), ("clusters", 50021, dict(M=64, k=64)),
                                       ("shared", 50021, dict(M=64, k=4)), ("dense", 50021, {}),
                                       ("clusters", 1 << 20, dict(M=4096, k=64))])
@pytest.mark.parametrize("where", [0.0, 0.5, 1.0])
def test_one_token_is_left_among_emptied_chunks(kind, V, kw, where):
    """The draft gives nothing to one token of p = 10^-11 and its share to all
    others, which are left nothing: whatever u, wherever it stands, that token is
    drawn, though rounding weighs the emptied chunks too."""
    B, allowed = 3, 400
    rng = np.random.default_rng(19)
    clusters = layout = None
    if kind == "dense":
        ids, cap = [np.arange(V)] * B, V
    else:
        of, layout = layout_of(V, kw["M"], 19)
        clusters = np.stack([rng.permutation(kw["M"])[:kw["k"]] for _ in range(B)]).astype(np.int32)
        shared = kind == "shared"
        ids = [shortlist(of, clusters.reshape(-1) if shared else c) for c in clusters]
        cap = D.union_cap(layout, B, kw["k"]) if shared else layout.cap(kw["k"])
    target = torch.full((B, 2, V), -math.inf)
    target[:, 1] = 0.0
    logits = np.full((B, cap), np.nan, dtype=np.float32)
    left = []
    for b in range(B):
        at = rng.permutation(len(ids[b]))[:allowed]
        at = at[np.argsort(ids[b][at])]
        z = rng.standard_normal(allowed).astype(np.float32)
        k = int(where * (allowed - 1))
        z[k] = -np.inf
        logits[b, :len(ids[b])] = -np.inf
        logits[b, at] = z
        z[k] = np.log(np.exp(z.astype(np.float64)).sum()) + math.log(1e-11)
        target[b, 0, torch.from_numpy(ids[b][at])] = torch.from_numpy(z)
        left.append(int(ids[b][at[k]]))
    tokens = torch.tensor([int(np.nonzero(np.isinf(f64(target[b, 0])))[0][0]) for b in range(B)], dtype=torch.int32)
    step = D.DraftStep(tokens.to(DEV), torch.zeros(B, device=DEV), torch.from_numpy(logits).to(DEV),
                       None if clusters is None else torch.from_numpy(clusters).to(DEV), shared=kind == "shared")
    for u in (0.0, 0.3, 1.0 - 2.0 ** -24):
        v = D.verify_chain(target.to(DEV), [step], torch.tensor([[0.75, u]]).repeat(B, 1).to(DEV), None, 1.0, layout)
        assert v.lengths.tolist() == [0] * B and v.ids[:, 0].tolist() == left
        for b in range(B):
            q = O.draft_distribution(V, logits[b].astype(np.float64), 1.0, ids[b])
            check(v, b, O.verify_chain(f64(target[b]), [int(tokens[b])], [0.75, u], 1, 1.0, lambda i: q, [1.0]), V)
