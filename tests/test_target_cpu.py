"""Host-side checks of the target's side: argument errors of the C ABI (no call
reaches a HIP API) and hand-worked pins of its oracle."""
import ctypes
import math

import numpy as np
import pytest

from oracle import target_oracle as O
from paper_2510_13847_amd import dynahead as D

P = 0x100000
BIG = 1 << 34


def _layout(V=1000, M=10):
    cap = (ctypes.c_int32 * (M + 1))(*([0] + [100 * (i + 1) for i in range(M)]))
    return D._Layout(V, 64, M, D.BF16, P, P, P, ctypes.addressof(cap), 100), cap


def _chain(n=2, B=2, V=1000, dtype=D.BF16, target=P, row=None, batch=None, steps=None, T=1.0, L=None, rows=P, u=P,
           ids=P, ws=P, nbytes=BIG):
    arr = (D._DraftStep * max(n, 1))(*(steps or [D._DraftStep(P, 0, 0, 0, 0, 0, 0, 0.0, 0.0)] * n))
    return D.lib().dyna_verify_chain(target, dtype, V, V if row is None else row, V * (n + 1) if batch is None else batch,
                                     B, n, arr, None, T, ctypes.byref(L) if L else None, rows, u, P, ids, P, ws, nbytes,
                                     None)


def test_chain_argument_errors():
    assert _chain(n=-1) == D.ERR_INVALID_ARG
    assert _chain(n=33, steps=[D._DraftStep(P)] * 33) == D.ERR_UNSUPPORTED
    assert _chain(V=0) == D.ERR_INVALID_ARG
    assert _chain(V=(1 << 22) + 1) == D.ERR_UNSUPPORTED
    assert _chain(B=-1) == D.ERR_INVALID_ARG
    assert _chain(B=1 << 23) == D.ERR_UNSUPPORTED           # more work items than one launch takes
    assert _chain(B=(1 << 21) + 1, n=1, V=8) == D.ERR_UNSUPPORTED  # requests: one workgroup of 1024 threads each
    assert _chain(dtype=2) == D.ERR_INVALID_ARG
    assert _chain(target=None) == D.ERR_INVALID_ARG
    assert _chain(target=P + 1) == D.ERR_INVALID_ARG
    assert _chain(row=999) == D.ERR_INVALID_ARG
    assert _chain(batch=10) == D.ERR_INVALID_ARG
    for T in (-0.5, float("inf"), float("nan"), 1e-40):     # (a denormal's reciprocal is no 32-bit number)
        assert _chain(T=T) == D.ERR_INVALID_ARG
    assert _chain(u=None) == D.ERR_INVALID_ARG
    assert _chain(ids=None) == D.ERR_INVALID_ARG
    assert _chain(ws=P + 8) == D.ERR_INVALID_ARG
    assert _chain(nbytes=64) == D.ERR_WORKSPACE
    assert _chain(B=0, target=None, ids=None, ws=None) == D.OK


def test_chain_step_errors():
    L, keep = _layout()
    ok = dict(tokens=P, logprobs=P, logits=P, clusters=P, k=3, cap=300, shared=0, temperature=1.0, tail_beta=0.0)

    def status(L=L, rows=P, **change):
        f = dict(ok, **change)
        return _chain(steps=[D._DraftStep(*[f[k] for k in ok])] * 2, L=L, rows=rows, nbytes=0)
    assert status() == D.ERR_WORKSPACE                      # everything else is in order
    assert status(tokens=None) == D.ERR_INVALID_ARG
    assert status(logprobs=None) == D.ERR_INVALID_ARG
    assert status(temperature=0.0) == D.ERR_INVALID_ARG
    assert status(temperature=1e-40) == D.ERR_INVALID_ARG
    assert status(tail_beta=1.0) == D.ERR_INVALID_ARG
    assert status(shared=2) == D.ERR_INVALID_ARG
    assert status(k=0) == D.ERR_INVALID_ARG
    assert status(k=11) == D.ERR_INVALID_ARG
    assert status(cap=299) == D.ERR_CAPACITY
    assert status(cap=599, shared=1) == D.ERR_CAPACITY      # two rows of up to 300
    assert status(L=None) == D.ERR_INVALID_ARG
    assert status(rows=None) == D.ERR_INVALID_ARG
    other, keep2 = _layout(V=900)
    assert status(L=other) == D.ERR_INVALID_ARG
    assert status(clusters=None, cap=1001) == D.ERR_INVALID_ARG
    assert status(clusters=None, tail_beta=0.1) == D.ERR_INVALID_ARG
    assert status(clusters=None, L=None, rows=None) == D.ERR_WORKSPACE
    assert D.lib().dyna_token_rows(ctypes.byref(L), P + 4, None) == D.ERR_INVALID_ARG
    assert D.lib().dyna_token_rows(None, P, None) == D.ERR_INVALID_ARG


def test_tree_argument_errors():
    def tree(N=5, V=1000, parents=P, stride=0, T=1.0, u=P, nodes=P, nbytes=0):
        return D.lib().dyna_verify_tree(P, D.F32, V, V, V * max(N, 1), 2, N, P, parents, stride, T, u, P, P, P, nodes,
                                        P, nbytes, None)
    assert tree() == D.ERR_WORKSPACE and tree(stride=5) == D.ERR_WORKSPACE and tree(nodes=None) == D.ERR_WORKSPACE
    assert tree(T=0.0, u=None) == D.ERR_WORKSPACE
    assert tree(N=0) == D.ERR_INVALID_ARG
    assert tree(N=1025) == D.ERR_UNSUPPORTED
    assert tree(parents=None) == D.ERR_INVALID_ARG
    assert tree(stride=4) == D.ERR_INVALID_ARG
    assert tree(u=None) == D.ERR_INVALID_ARG
    assert D.lib().dyna_verify_workspace_bytes(0, 5, 100, 0) == 0
    assert D.lib().dyna_verify_workspace_bytes(1, 5, 100, 0) > 0


def test_distill_argument_errors():
    lib = D.lib()

    def call(logits=P, dtype=D.BF16, V=1000, row=1000, N=4, ids=P, values=P, vdtype=D.F32, K=8, tail=0, T=1.0, loss=P,
             grad=BIG, grow=1000, ws=P, nbytes=0):
        return lib.dyna_distill(logits, dtype, V, row, N, ids, values, vdtype, K, tail, T, None, loss, None, grad, grow,
                                ws, nbytes, None)
    assert call() == D.ERR_WORKSPACE and call(grad=None, grow=0) == D.ERR_WORKSPACE
    assert call(N=0, logits=None, ids=None) == D.OK
    for bad in (dict(logits=None), dict(logits=P + 1), dict(dtype=5), dict(vdtype=5), dict(V=0), dict(row=999),
                dict(N=-1), dict(ids=None), dict(values=None), dict(K=0), dict(tail=2), dict(T=0.0),
                dict(T=float("nan")), dict(loss=None), dict(grow=999), dict(ws=None), dict(grad=P),
                dict(grad=P + 7000)):
        assert call(**bad) == D.ERR_INVALID_ARG, bad
    assert call(K=1025) == D.ERR_UNSUPPORTED
    assert call(V=1 << 23, row=1 << 23, grow=1 << 23) == D.ERR_UNSUPPORTED
    back = lib.dyna_distill_grad
    assert back(P, D.BF16, 1000, 1000, 4, P, P, D.F32, 8, 0, 1.0, None, None, BIG, 1000, None) == D.ERR_INVALID_ARG
    assert back(P, D.BF16, 1000, 1000, 4, P, P, D.F32, 8, 0, 1.0, None, P, None, 1000, None) == D.ERR_INVALID_ARG
    assert back(P, D.BF16, 1000, 1000, 0, None, None, D.F32, 8, 0, 1.0, None, None, None, 0, None) == D.OK


def test_router_loss_argument_errors():
    def call(scores=P, dtype=D.F32, M=100, row=100, N=4, ids=P, L=8, of=P, V=1000, pw=1.0, loss=P, grad=None, grow=0):
        return D.lib().dyna_router_loss(scores, dtype, M, row, N, ids, L, of, V, pw, None, loss, grad, grow, None)
    for bad in (dict(scores=None), dict(dtype=7), dict(M=0), dict(row=99), dict(N=-1), dict(ids=None), dict(of=None),
                dict(V=0), dict(pw=0.0), dict(pw=float("nan")), dict(loss=None), dict(grad=P + 400, grow=100),
                dict(grad=P, grow=101), dict(grad=BIG, grow=99), dict(L=-1)):
        assert call(**bad) == D.ERR_INVALID_ARG, bad
    assert call(M=8193, row=8193) == D.ERR_UNSUPPORTED
    assert call(L=1025) == D.ERR_UNSUPPORTED
    assert call(N=0, scores=None) == D.OK


# ---------------------------------------------------------------- the oracle by hand
LN = math.log


def test_oracle_chain_by_hand():
    # p = (1/2, 1/4, 1/4) in every row; the draft gives token 0 everything
    target = np.log(np.array([[2.0, 1.0, 1.0]] * 3))
    q = np.array([1.0, 0.0, 0.0])
    run = lambda tok, u, **kw: O.verify_chain(target, tok, u, 2, 1.0, **kw)[:2]
    # u q < p: 0.4 < 0.5 stands, 0.6 falls; the residual is (0, 1/4, 1/4)
    dist = dict(q_of=lambda i: q, q_token=[1.0, 1.0])
    assert run([0, 0], [0.4, 0.6, 0.49], **dist) == (1, [0, 1])
    assert run([0, 0], [0.4, 0.6, 0.5], **dist) == (1, [0, 2])
    assert run([0, 0], [0.4, 0.4, 0.49], **dist) == (2, [0, 0, 0])
    # outright at token 1: falls at u = 0.3; the rest is (1/2, 0, 1/4)
    assert run([1, 0], [0.3, 0.0, 0.66]) == (0, [0])
    assert run([1, 0], [0.3, 0.0, 0.67]) == (0, [2])
    # no token: drawn from p itself
    assert run([-1, 0], [0.0, 0.0, 0.74]) == (0, [1])
    assert O.verify_chain(target, [0, 2], [0, 0, 0], 2, 0.0)[:2] == (1, [0, 0])


def test_oracle_tree_by_hand():
    row = np.log(np.array([4.0, 2.0, 1.0, 1.0]) / 8)
    target = np.stack([row] * 4)
    run = lambda tok, par, u: O.verify_tree(target, tok, par, u, 1.0)
    # child 0 falls (0.5 >= 1/2), child 1 is tested with 1/4 over 1/2: 0.49 stands, then a leaf
    n, ids, _, nodes = run([9, 0, 1, 2], [0, 0, 0, 0], [0.51, 0.5, 0.49, 0.0])
    assert (n, ids, nodes) == (1, [1, 1], [2])
    # both fall, and the third: the rest is token 3
    n, ids, _, nodes = run([9, 0, 1, 2], [0, 0, 0, 0], [0.0, 0.6, 0.6, 0.6])
    assert (n, ids, nodes) == (0, [3], [])
    # an equal sibling has nothing left
    n, ids, _, nodes = run([9, 0, 0, 1], [0, 0, 0, 2], [0.0, 0.6, 0.0, 0.0])
    assert (n, ids, nodes) == (0, [1], [])


def test_oracle_distillation_by_hand():
    z = np.array([LN(4.0), LN(2.0), LN(1.0), LN(1.0)])  # q = 1/2, 1/4, 1/8, 1/8
    loss, grad, (lse, rest), _ = O.distill_row(z, [1, 0], [LN(0.25), LN(0.25)], 1.0, True)
    # p = 1/4 on each of tokens 0 and 1, 1/2 left against q's 1/4 there
    assert abs(loss - (0.25 * LN(0.5) + 0.25 * LN(1.0) + 0.5 * LN(2.0))) < 1e-15
    assert np.allclose(grad, [0.25, 0.0, -0.125, -0.125], atol=1e-15)
    assert abs(lse - LN(8.0)) < 1e-15 and abs(rest - LN(2.0)) < 1e-15
    loss, grad, _, _ = O.distill_row(z, [1, 0, 1, -1], [0.0, 0.0, 9.0, 9.0], 1.0, False)
    assert abs(loss - 0.5 * (LN(1.0) + LN(2.0))) < 1e-15
    assert np.allclose(grad, [0.0, -0.25, 0.125, 0.125], atol=1e-15)


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    z, ids, t = rng.standard_normal(9), [3, 0, 7], np.log([0.3, 0.2, 0.1])
    for tail in (False, True):
        grad = O.distill_row(z, ids, t, 0.7, tail)[1]
        for v in range(9):
            e = np.zeros(9)
            e[v] = 1e-5
            d = (O.distill_row(z + e, ids, t, 0.7, tail)[0] - O.distill_row(z - e, ids, t, 0.7, tail)[0]) / 2e-5
            assert abs(d - grad[v]) < 1e-9
    s, y = rng.standard_normal(6), np.array([1, 0, 0, 1, 0, 1], dtype=bool)
    grad = O.router_row(s, y, 3.0)[1]
    for m in range(6):
        e = np.zeros(6)
        e[m] = 1e-5
        assert abs((O.router_row(s + e, y, 3.0)[0].sum() - O.router_row(s - e, y, 3.0)[0].sum()) / 2e-5 - grad[m]) < 1e-9


def test_a_mistaken_oracle_is_seen():
    """Planted mistakes change a result: dividing the tree's test by nothing,
    drawing a fallen chain from p, leaving the tail out of the gradient."""
    row = np.log(np.array([4.0, 2.0, 1.0, 1.0]) / 8)
    p = O.softmax(row, 1.0)
    assert not (0.49 < p[1]) and 0.49 * (1 - p[0]) < p[1]
    assert O.place(np.maximum(p - np.array([1.0, 0, 0, 0]), 0), 0.1) != O.place(p, 0.1)
    a = O.distill_row(row, [0], [LN(0.25)], 1.0, True)[1]
    b = O.distill_row(row, [0], [LN(0.25)], 1.0, False)[1]
    assert np.abs(a - b).max() > 0.1


@pytest.mark.parametrize("T", [1e-46, -1e-46, 5e-324])
def test_a_temperature_that_32_bits_round_to_zero_is_refused(T):
    """The library takes 0 as greedy verification; only 0 itself asks for it."""
    assert ctypes.c_float(T).value == 0.0
    for make in (lambda: D.ChainVerifier(1, 1, 8, T, device="cpu"), lambda: D.TreeVerifier(1, 2, 8, T, device="cpu")):
        with pytest.raises(ValueError, match="32 bits"):
            make()
    for ok in (0.0, 1.0, float(np.float32(1.2e-38))):
        assert D.ChainVerifier(1, 1, 8, ok, device="cpu").temperature == ok


def test_a_layout_on_another_device_is_refused():
    """Its tables would be read by kernels on the verifier's device."""
    import types

    import torch
    layout = types.SimpleNamespace(M=4, V=8, perm=torch.empty(8, dtype=torch.int32, device="meta"))
    with pytest.raises(ValueError, match="layout is on meta"):
        D.ChainVerifier(1, 1, 8, layout=layout, device="cpu")
