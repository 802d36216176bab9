"""The target's side as it is used next to the draft head.

A cycle of chain drafting: a DraftHead per position, each with its own cluster
budget, sampling; the target's rows from a DenseHead; the chain judged.  A tree
grown by beam expansion and judged.  The target's top list from a DenseHead,
and from it the drafter's and the router's losses and gradients.  Every result
is checked against the fp64 oracle on the device's own upstream values."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from oracle import target_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = None
V, DIM, M = 6001, 256, 60


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


def model(B):
    w = W.scaled(W.WORKLOADS["llama3_8b_chain"], name="target_cycle", V=V, d=DIM, M=M, H=64, B=B)
    of = W.partition(w)
    W_lm = (2.5 * W.lm_head(w, "cpu")).to(torch.bfloat16).to(DEV)
    W1, W2 = W.router_weights(w, "cpu")
    layout = D.build_layout(torch.from_numpy(of).to(DEV), W_lm, M)
    return w, of, W_lm, layout, D.Router(W1.to(DEV), W2.to(DEV), act=w.act)


def rows_like(h, seed):
    """Target hidden rows: the drafter's with an error of their own."""
    g = torch.Generator().manual_seed(seed)
    return (h.float() + 0.5 * torch.randn(h.shape, generator=g).to(DEV)).to(torch.bfloat16)


@pytest.mark.parametrize("B,tail,union", [(1, 0.0, False), (5, 0.0, False), (4, 0.125, False), (3, 0.0, True)])
def test_drafted_chain_is_judged(B, tail, union):
    w, of, W_lm, layout, router = model(B)
    n, T = 4, 0.75
    mode = D.SEL_SAMPLE | (D.SEL_UNION if union else 0)
    heads, hidden = [], []
    for i in range(n):
        k = D.cluster_budget(i, 16, 12, 2)
        h = W.contexts(w, DEV, batch=B, salt=i)
        head = D.DraftHead(router, layout, B, k, mode, temperature=T, keep_logits=True, tail_beta=tail)
        head(h, h, W.uniforms(w, DEV, batch=B, salt=i))
        heads.append(head)
        hidden.append(h)
    hidden.append(W.contexts(w, DEV, batch=B, salt=n))
    rows = torch.stack([rows_like(h, i) for i, h in enumerate(hidden)], 1).reshape(B * (n + 1), DIM).contiguous()
    dense = D.DenseHead(W_lm, V, B * (n + 1), D.SEL_ARGMAX, keep_logits=True)
    target = dense(rows).logits.view(B, n + 1, V)
    u = torch.rand((B, n + 1), generator=torch.Generator().manual_seed(B)).to(DEV)
    steps = [D.DraftStep.of(h) for h in heads]
    v = D.ChainVerifier(B, n, V, T, layout)(target, steps, u)
    greedy = D.verify_chain(target, [D.DraftStep(h.sample) for h in heads], None, None, 0.0)
    zs, us, stood = f64(target), f64(u), 0
    for b in range(B):
        def q_of(i):
            cl = heads[i].clusters.cpu().numpy()
            ids = np.concatenate([np.nonzero(of == m)[0] for m in sorted(set((cl if union else cl[b]).reshape(-1)))])
            return O.draft_distribution(V, f64(heads[i].logits[b]), T, ids, tail)
        tokens = [int(h.sample[b]) for h in heads]
        for i in range(n):  # the head's own report of its sample agrees with its logits
            assert abs(math.log(q_of(i)[tokens[i]]) - float(heads[i].sample_logprob[b])) < 1e-4
        a, ids, lps = O.verify_chain(zs[b], tokens, us[b], n, T, q_of,
                                     [math.exp(float(h.sample_logprob[b])) for h in heads])
        assert int(v.lengths[b]) == a and v.ids[b].tolist() == ids + [-1] * (n + 1 - len(ids))
        stood += a
        a, ids, _ = O.verify_chain(zs[b], tokens, us[b], n, 0.0)
        assert int(greedy.lengths[b]) == a and greedy.ids[b].tolist() == ids + [-1] * (n + 1 - len(ids))
    assert stood > 0 or B == 1


def test_beam_tree_is_judged():
    """Levels of beam expansion become a tree: node (level, rank), its parent the
    beam row it extends.  The target judges it in one call."""
    width, depth = 6, 3
    w, of, W_lm, layout, router = model(1)
    h = W.contexts(w, DEV, batch=1)
    tokens, parents, rows, last = [torch.zeros(1, dtype=torch.int32, device=DEV)], [0], [rows_like(h, 50)], None
    first = 0
    hb = h
    for t in range(depth):
        head = D.DraftHead(router, layout, hb.shape[0], 12, D.SEL_TOPK | (D.SEL_UNION if t else 0), width,
                           keep_logits=False)
        head(hb, hb)
        last, parent, ids = D.beam_expand(head.logprobs, head.ids, last if t else None, width)
        tokens.append(ids)
        parents += [first + p if t else 0 for p in parent.tolist()]
        first = 1 if not t else first + width
        hb = (hb[parent.long()].float() * 0.5 + W_lm[ids.long()].float() * 20.0).to(torch.bfloat16)
        rows.append(rows_like(hb, 60 + t))
    tokens = torch.cat(tokens)[None].contiguous()
    N = tokens.shape[1]
    dense = D.DenseHead(W_lm, V, N, D.SEL_ARGMAX, keep_logits=True)
    target = dense(torch.cat(rows).contiguous()).logits.view(1, N, V)
    par = torch.tensor(parents, dtype=torch.int32, device=DEV)
    ver = D.TreeVerifier(1, N, V, 1.0)
    deepest = 0
    for seed in range(20):
        u = torch.rand((1, N), generator=torch.Generator().manual_seed(seed)).to(DEV)
        u[:, 1:] *= 0.25
        ver(target, tokens, par, u)
        a, ids, _, nodes = O.verify_tree(f64(target)[0], tokens[0].tolist(), parents, f64(u)[0], 1.0)
        assert int(ver.lengths[0]) == a and ver.ids[0].tolist() == ids + [-1] * (N - len(ids))
        assert ver.nodes[0].tolist() == nodes + [-1] * (N - len(nodes))
        deepest = max(deepest, a)
    assert deepest >= 1


def test_target_teaches_drafter_and_router():
    """The target's top 16 of each row, as a DenseHead reports them, train a
    student's hidden rows and a router: losses and gradients, taken on through
    torch's products, against the oracle's."""
    N, K, T = 7, 16, 1.0
    w, of, W_lm, layout, router = model(N)
    teacher = D.DenseHead(W_lm, V, N, D.SEL_TOPK, K)
    h = W.contexts(w, DEV, batch=N)
    teacher(rows_like(h, 80))
    weights = torch.full((N,), 1.0 / (N - 1), device=DEV)
    weights[-1] = 0.0
    x = h.float().requires_grad_(True)
    logits = x @ W_lm.float().t()
    loss, stats, grad = D.distill(logits.detach(), teacher.ids, teacher.logprobs, T, True, weights, want_stats=True)
    logits.backward(grad)
    ids, values, z = teacher.ids.cpu().numpy(), f64(teacher.logprobs), f64(logits)
    want = np.zeros((N, V))
    for r in range(N - 1):
        l, g, _, _ = O.distill_row(z[r], ids[r], values[r], T, True)
        want[r] = g * float(weights[r])
        assert abs(float(loss[r]) - l) < 1e-5
    dx = want @ f64(W_lm)
    # gradients of up to 1/6, errors of 1e-6 of them, through sums of 6001 products with W of size 0.16
    assert np.abs(f64(x.grad) - dx).max() < 1e-5 * max(1.0, np.abs(dx).max())
    assert not x.grad[-1].any()

    W1, W2 = router.W1.float().requires_grad_(True), router.W2.float().requires_grad_(True)
    hid = torch.nn.functional.silu(h.float() @ W1.t())
    scores = hid @ W2.t()
    _, _, ours = D.route(router, h, 4, want_scores=True)
    assert (ours - scores).abs().max() < 2e-3  # the library's scores of the same router
    rloss, rgrad = D.router_loss(scores.detach(), teacher.ids, torch.from_numpy(of).to(DEV), 4.0, weights)
    scores.backward(rgrad)
    labels = torch.zeros((N, M), dtype=torch.bool)
    for r in range(N):
        labels[r, of[ids[r]].tolist()] = True
    ref = torch.nn.functional.binary_cross_entropy_with_logits(
        scores.detach().double().cpu(), labels.double(), reduction="none", pos_weight=torch.full((M,), 4.0).double())
    assert (rloss.cpu().double() - ref.sum(1) * (weights.cpu() != 0)).abs().max() < 1e-4
    a1, a2 = router.W1.float().requires_grad_(True), router.W2.float().requires_grad_(True)
    s = torch.nn.functional.silu(h.float() @ a1.t()) @ a2.t()
    cost = torch.nn.functional.binary_cross_entropy_with_logits(
        s, labels.to(DEV).float(), reduction="none", pos_weight=torch.full((M,), 4.0, device=DEV))
    (cost.sum(1) * weights).sum().backward()
    for got, exp in ((W1.grad, a1.grad), (W2.grad, a2.grad)):
        assert (got - exp).abs().max() <= 1e-5 * exp.abs().max()


def head_of(kind, w, layout, router, W_lm, B, T):
    sampled = dict(temperature=T, keep_logits=True)
    if kind == "dense":
        return D.DenseHead(W_lm, V, B, D.SEL_SAMPLE, **sampled)
    if kind == "union":
        return D.DraftHead(router, layout, B, 3, D.SEL_SAMPLE | D.SEL_UNION, **sampled)
    if kind == "argmax":
        return D.DraftHead(router, layout, B, 8, D.SEL_ARGMAX)
    if kind == "best of 4":
        return D.DraftHead(router, layout, B, 8, D.SEL_TOPK, 4)
    return D.DraftHead(router, layout, B, 8, D.SEL_SAMPLE, tail_beta=0.125 if kind == "tail" else 0.0, **sampled)


KINDS = ["shortlist", "tail", "union", "dense", "argmax", "best of 4"]


@pytest.mark.parametrize("kind", KINDS)
def test_one_head_drafts_position_after_position(kind):
    """A step is what its head wrote at that position, though the head ran again:
    the chain is judged as one drafted by a head for each position, also where the
    steps are taken on a side stream and inside a captured graph."""
    B, n, T = 6, 4, 0.75
    w, of, W_lm, layout, router = model(B)
    hidden = [W.contexts(w, DEV, batch=B, salt=i) for i in range(n + 1)]
    us = [W.uniforms(w, DEV, batch=B, salt=i) for i in range(n)]
    rows = torch.stack([rows_like(h, i) for i, h in enumerate(hidden)], 1).reshape(B * (n + 1), DIM).contiguous()
    target = D.DenseHead(W_lm, V, B * (n + 1), D.SEL_ARGMAX, keep_logits=True)(rows).logits.view(B, n + 1, V)
    u = 0.2 * torch.rand((B, n + 1), generator=torch.Generator().manual_seed(4)).to(DEV)

    def run(head, i, **kw):
        return head(hidden[i], us[i], **kw) if kind == "dense" else head(hidden[i], hidden[i], us[i], **kw)

    def results(v):
        return [x.clone() for x in (v.lengths, v.ids, v.logprobs)]
    heads = [run(head_of(kind, w, layout, router, W_lm, B, T), i) for i in range(n)]
    ver = D.ChainVerifier(B, n, V, T, layout)
    want = results(ver(target, [D.DraftStep.of(h) for h in heads], u))
    assert int(want[0].max()) > 0
    one = head_of(kind, w, layout, router, W_lm, B, T)
    got = results(ver(target, [D.DraftStep.of(run(one, i)) for i in range(n)], u))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    steps = [D.DraftStep.of(run(one, i, stream=side), stream=side) for i in range(n)]
    ver(target, steps, u, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results(ver), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps = [D.DraftStep.of(run(one, i)) for i in range(n)]
        ver(target, steps, u)
    for again in range(3):
        ver.ids.fill_(-7)
        run(one, again)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(ver), want))


@pytest.mark.parametrize("kind", KINDS)
def test_a_head_that_has_not_run_has_no_step(kind):
    w, of, W_lm, layout, router = model(2)
    with pytest.raises(ValueError, match="has not run"):
        D.DraftStep.of(head_of(kind, w, layout, router, W_lm, 2, 1.0))
