"""Distillation from a teacher's top list and the router's loss, against the
fp64 oracle and against differences.

Error bounds (u = 2^-24).  The exponentials of a row err by (2.9 x + 2) u for
logits x below the largest over T (two roundings of x log2(e), one of the
exponential), a row's sum by the mean of that, at most (2.9 ln V + 9) u with
the fp32 sum of eight.  So the loss, whose logs carry that twice, is within
2 (2.9 ln V + 16) u plus its own rounding, and an element of the gradient within
(2.9 x + 2 * 2.9 ln V + 32) u of the sum of the sizes of its terms, plus the
rounding to its type, half an eps.  The router's terms k softplus and k sigma
err by (1.5 |s| + 16) u of themselves.
"""
import math

import numpy as np
import pytest
import torch

from oracle import target_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
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


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def problem(N, V, K, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    logits = (spread * torch.randn((N, V), generator=g)).to(DT[dtype])
    z = 0.7 * logits.float() + 2.0 * torch.randn((N, V), generator=g)
    k = min(K, V)
    top = z.topk(k, 1)
    ids = torch.full((N, K), -1, dtype=torch.int32)
    values = torch.zeros((N, K))
    ids[:, :k] = top.indices
    values[:, :k] = top.values - torch.logsumexp(z, 1, keepdim=True)
    return logits, ids, values


def check_rows(logits, ids, values, T, tail, weights, loss, stats, grad, rows=None):
    V = logits.shape[1]
    T = float(np.float32(T))
    zs, ii, vv = f64(logits), ids.cpu().numpy(), f64(values)
    lg = 2.9 * math.log(max(V, 2))
    for r in range(logits.shape[0]) if rows is None else rows:
        w = 1.0 if weights is None else float(weights[r])
        if w == 0.0:
            assert loss is None or float(loss[r]) == 0.0
            assert grad is None or not grad[r].any()
            continue
        want, g, lse, size = O.distill_row(zs[r], ii[r], vv[r], T, tail)
        if loss is not None:
            got = float(loss[r])
            assert got == want or abs(got - want) <= 2 * (lg + 16) * U + abs(want) * U, (r, got, want)
        if stats is not None:
            for a, b in zip(f64(stats[r]), lse):
                assert a == b or abs(a - b) <= (lg + 16) * U + abs(b) * 2.0 ** -50, (r, a, b)
        if grad is not None:
            finite = zs[r][np.isfinite(zs[r])]
            x = (finite.max() if finite.size else 0.0) - zs[r]
            with np.errstate(invalid="ignore"):
                near = np.where(size > 0, (2.9 * np.minimum(x / T, 200.0) + 2 * lg + 32) * U * size, 0.0)
            tol = abs(w) * (near + np.abs(g) * torch.finfo(grad.dtype).eps / 2) + 1e-37
            off = np.abs(f64(grad[r]) - w * g)
            assert (off <= tol).all(), (r, int((off - tol).argmax()), off.max(), f64(grad[r])[(off - tol).argmax()],
                                        (w * g)[(off - tol).argmax()])


SHAPES = [  # N, V, K, dtype, T, tail
    (1, 1, 1, "f32", 1.0, False), (2, 1, 1, "bf16", 1.0, True), (3, 5, 5, "f32", 1.0, True),
    (3, 7, 2, "bf16", 2.0, False), (4, 2047, 8, "bf16", 1.0, True), (5, 2048, 64, "f32", 0.7, False),
    (7, 2049, 33, "f32", 1.0, True), (1, 50021, 64, "bf16", 1.0, True), (33, 4099, 1, "bf16", 1.5, False),
    (3, 131077, 16, "bf16", 1.0, False), (2, 262144, 1024, "f32", 2.0, True), (2, 1500, 1024, "f32", 1.0, False),
    (2300, 520, 10, "bf16", 1.0, True), (300, 66001, 5, "bf16", 1.0, True), (513, 8200, 40, "f32", 1.0, False),
]


@pytest.mark.parametrize("N,V,K,dtype,T,tail", SHAPES)
def test_distill(N, V, K, dtype, T, tail):
    logits, ids, values = problem(N, V, K, dtype, N + V + K)
    g = torch.Generator().manual_seed(1)
    weights = torch.rand(N, generator=g) + 0.1
    weights[torch.rand(N, generator=g) < 0.2] = 0.0
    weights[0] = -0.5 if N > 1 else 1.0
    dev = [x.to(DEV) for x in (logits, ids, values, weights)]
    loss, stats, grad = D.distill(dev[0], dev[1], dev[2], T, tail, dev[3], want_stats=True)
    rows = sorted(set(list(range(min(N, 6))) + [N // 2, N - 1]))
    check_rows(logits, ids, values, T, tail, weights, loss, stats, grad, rows)
    # the loss alone, and the gradient alone from the forward pass's statistics
    only, none, no = D.distill(dev[0], dev[1], dev[2], T, tail, dev[3], want_grad=False)
    assert none is None and no is None
    check_rows(logits, ids, values, T, tail, weights, only, None, None, rows)
    back = D.distill_grad(dev[0], stats, dev[1], dev[2], T, tail, dev[3])
    check_rows(logits, ids, values, T, tail, weights, None, None, back, rows)


EDGES = [  # N, V, K, dtype: rows and lists at and just behind what a kernel's registers and threads hold
    (200, 1020, 4, "f32"), (1100, 1024, 4, "f32"), (1100, 2055, 300, "bf16"), (170, 8192, 256, "f32"),
    (170, 8193, 257, "f32"), (165, 16384, 256, "f32"), (165, 16388, 255, "f32"), (165, 32768, 256, "bf16"),
    (165, 40007, 20, "bf16"), (165, 20003, 300, "f32"), (165, 65536, 512, "bf16"), (165, 65543, 513, "bf16"),
    (260, 131072, 600, "bf16"), (165, 131080, 64, "bf16"), (161, 65539, 1024, "f32"), (40000, 5, 2, "f32"),
]


@pytest.mark.parametrize("N,V,K,dtype", EDGES)
def test_distill_at_the_edges_of_its_kernels(N, V, K, dtype):
    logits, ids, values = problem(min(N, 40), V, K, dtype, N + V + K)
    pick = torch.arange(N) * 7 % logits.shape[0]      # rows repeat: each is held to its own place's result
    logits, ids, values = logits[pick], ids[pick], values[pick]
    weights = torch.where(torch.arange(N) % 5 == 1, 0.0, 0.5 + torch.arange(N) / N)
    weights[N - 3:] = 0.0
    dev = [x.to(DEV) for x in (logits, ids, values, weights)]
    loss, stats, grad = D.distill(dev[0], dev[1], dev[2], 1.0, True, dev[3], want_stats=True)
    rows = sorted({0, 1, 2, N // 3, N // 2, N - 4, N - 3, N - 1})
    check_rows(logits, ids, values, 1.0, True, weights, loss, stats, grad, rows)
    # the same row has the same loss wherever it stands
    live = weights != 0
    first = torch.full((int(pick.max()) + 1,), -1, dtype=torch.long)
    for i in reversed(torch.nonzero(live).flatten().tolist()):
        first[pick[i]] = i
    assert torch.equal(loss.cpu()[live], loss.cpu()[first[pick]][live])
    assert not loss.cpu()[~live].any() and not grad[(~live).to(DEV)].any()
    # nothing but padding
    loss, stats, grad = D.distill(dev[0], dev[1], dev[2], 1.0, True, torch.zeros_like(dev[3]), want_stats=True)
    assert not loss.any() and not stats.any() and not grad.any()


@pytest.mark.parametrize("tail", [False, True])
def test_distill_lists_with_repeats_and_strangers(tail):
    """Ids outside the vocabulary and ids that stood earlier in the row are no
    entries, whatever their values; a row without any entry is still."""
    N, V, K = 6, 3001, 40
    logits, ids, values = problem(N, V, K, "f32", 5)
    values = values - 1.0
    ids[1, 5:20] = ids[1, 3]
    ids[2, ::2] = -1
    ids[2, 1::4] = V
    ids[3, :] = -7
    ids[4, :] = 17
    values[4, 1:] = math.inf                       # not read: repeats
    ids[5, 0], values[5, 0] = V - 1, -math.inf     # an entry the teacher gives nothing
    dev = [x.to(DEV) for x in (logits, ids, values)]
    loss, stats, grad = D.distill(*dev, 1.0, tail, want_stats=True)
    check_rows(logits, ids, values, 1.0, tail, None, loss, stats, grad)
    check_rows(logits, ids, values, 1.0, tail, None, None, None, D.distill_grad(dev[0], stats, *dev[1:], 1.0, tail))
    assert float(loss[3]) == 0.0 and (tail or not grad[3].any())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_masked_students(tail, dtype):
    """-inf and the type's lowest value in the student's rows: on the list, off
    it, everywhere but the list, everywhere."""
    N, V, K = 7, 4097, 6
    logits, ids, values = problem(N, V, K, dtype, 6)
    low = torch.finfo(DT[dtype]).min
    logits[0, ids[0, 2].long()] = -math.inf        # q = 0 where p > 0: loss +inf
    logits[1, 1000:] = -math.inf
    logits[1, ids[1].long()] = 1.0
    logits[2] = -math.inf
    logits[2, ids[2].long()] = 0.5                 # nothing outside the list
    logits[3] = -math.inf                          # nothing at all
    logits[4] = low
    logits[5, 50:] = low
    logits[5, ids[5].long()] = 0.0
    logits[6] = -200.0                             # a rest 2^-288 below the list
    logits[6, ids[6].long()] = torch.arange(K, dtype=torch.float32).to(DT[dtype])
    dev = [x.to(DEV) for x in (logits, ids, values)]
    loss, stats, grad = D.distill(*dev, 1.0, tail, want_stats=True)
    assert torch.isfinite(grad.float()).all()
    check_rows(logits, ids, values, 1.0, tail, None, loss, stats, grad)
    back = D.distill_grad(dev[0], stats, *dev[1:], 1.0, tail)
    check_rows(logits, ids, values, 1.0, tail, None, None, None, back)


@pytest.mark.parametrize("T", [1e-20, 1e20])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N", [5, 170])
def test_distill_temperatures_at_their_ends(N, tail, T):
    """One-hot and flat students and teachers, by either kernel."""
    V, K = 9001, 12
    logits, ids, values = problem(5, V, K, "f32", 21)
    logits[1] = 0.0
    pick = torch.arange(N) % 5
    logits, ids, values = logits[pick], ids[pick], values[pick]
    dev = [x.to(DEV) for x in (logits, ids, values)]
    loss, stats, grad = D.distill(*dev, T, tail, want_stats=True)
    rows = [0, 1, 2, 3, 4, N - 1]
    check_rows(logits, ids, values, T, tail, None, loss, stats, grad, rows)
    check_rows(logits, ids, values, T, tail, None, None, None, D.distill_grad(dev[0], stats, *dev[1:], T, tail), rows)


def test_distill_undefined_rows_show():
    N, V, K = 5, 2500, 4
    logits, ids, values = problem(N, V, K, "f32", 7)
    logits[0, 1234] = math.nan
    logits[1, 3] = math.inf
    logits[2, ids[2, 1].long()] = math.nan
    values[3, 2] = math.nan
    for tail in (False, True):
        dev = [x.to(DEV) for x in (logits, ids, values)]
        loss, _, grad = D.distill(*dev, 1.0, tail)
        assert loss[:4].isnan().all() and grad[:4].isnan().all(dim=1).all()
        check_rows(logits, ids, values, 1.0, tail, None, loss, None, grad, rows=[4])


def test_distill_padding_is_not_read_and_neighbours_stay():
    """Rows inside larger buffers at odd offsets; padding rows full of NaN with
    wild ids; the memory around the gradient's rows keeps its values."""
    N, V, K = 9, 2053, 5
    for dtype in ("f32", "bf16"):
        logits, ids, values = problem(N, V, K, dtype, 8)
        weights = torch.full((N,), 0.25)
        weights[6:] = 0.0
        big = torch.full((N, V + 7), math.nan, dtype=DT[dtype])
        big[:6, 3:V + 3] = logits[:6]
        ids[6:] = 2 ** 31 - 1
        values[6:] = math.nan
        out = torch.full((N, V + 9), 7.0, dtype=DT[dtype], device=DEV)
        side = torch.cuda.Stream()
        dev = [x.to(DEV) for x in (big, ids, values, weights)]
        torch.cuda.synchronize()
        loss, _, grad = D.distill(dev[0][:, 3:V + 3], dev[1], dev[2], 1.0, True, dev[3], out=out[:, 5:V + 5],
                                  stream=side)
        side.synchronize()
        check_rows(logits, ids, values, 1.0, True, weights, loss, None, grad)
        assert (out[:, :5] == 7.0).all() and (out[:, V + 5:] == 7.0).all()


def test_distill_rows_beyond_32_bit_offsets():
    V, K = 5001, 4
    stride = (1 << 31) + 333
    logits, ids, values = problem(2, V, K, "bf16", 9)
    buf = torch.zeros(stride + V, dtype=torch.bfloat16, device=DEV)
    gbuf = torch.zeros(stride + V, dtype=torch.bfloat16, device=DEV)
    z, out = (torch.as_strided(x, (2, V), (stride, 1)) for x in (buf, gbuf))
    z.copy_(logits)
    loss, _, grad = D.distill(z, ids.to(DEV), values.to(DEV), out=out)
    check_rows(logits, ids, values, 1.0, False, None, loss, None, grad)


def test_distill_gradient_against_differences():
    """Central differences of the kernel's own fp32 loss.  With h = 2^-5 its error
    is the loss's, about 40 u over 2h = 4e-5, and h^2 / 6 of the third derivative,
    at most 1/6 of q_v: 3e-5."""
    N, V, K = 1, 700, 12
    logits, ids, values = problem(N, V, K, "f32", 10, spread=1.0)
    h = 2.0 ** -5
    for tail in (False, True):
        _, _, grad = D.distill(logits.to(DEV), ids.to(DEV), values.to(DEV), 1.0, tail)
        for v in list(ids[0, :4].tolist()) + [0, 350, 699]:
            two = logits.repeat(2, 1)
            two[0, v] += h
            two[1, v] -= h
            loss, _, _ = D.distill(two.to(DEV), ids.repeat(2, 1).to(DEV), values.repeat(2, 1).to(DEV), 1.0, tail,
                                   want_grad=False)
            d = (float(loss[0]) - float(loss[1])) / float(two[0, v].double() - two[1, v].double())
            assert abs(d - float(grad[0, v])) <= 8e-5, (tail, v, d, float(grad[0, v]))


def test_teacher_values_in_bf16():
    logits, ids, values = problem(4, 3000, 20, "bf16", 12)
    values = values.to(torch.bfloat16)
    loss, _, grad = D.distill(logits.to(DEV), ids.to(DEV), values.to(DEV), 0.5)
    check_rows(logits, ids, values, 0.5, False, None, loss, None, grad)


@pytest.mark.parametrize("N,M,L,dtype,pw", [
    (1, 1, 1, "f32", 1.0), (3, 7, 4, "bf16", 2.5), (5, 64, 8, "f32", 1.0), (4, 1023, 64, "bf16", 8.0),
    (3, 4096, 100, "f32", 8.0), (2, 8192, 1024, "bf16", 1.0), (2, 8191, 3, "f32", 0.5), (600, 200, 10, "f32", 1.0)])
def test_router_loss(N, M, L, dtype, pw):
    V = 9000
    g = torch.Generator().manual_seed(N + M + L)
    scores = (4.0 * torch.randn((N, M), generator=g) - 3.0).to(DT[dtype])
    scores[0, 0] = -100.0
    scores[-1, -1] = 90.0
    of = torch.randint(0, M, (V,), generator=g, dtype=torch.int32)
    ids = torch.randint(0, V, (N, L), generator=g, dtype=torch.int32)
    ids[:, L // 2] = -1
    if L > 3:
        ids[0, 1], ids[0, 2] = V, ids[0, 0]
    weights = torch.rand(N, generator=g)
    if N > 2:
        weights[1] = 0.0
    dev = [x.to(DEV) for x in (scores, ids, of, weights)]
    loss, grad = D.router_loss(dev[0], dev[1], dev[2], pw, dev[3])
    only, none = D.router_loss(dev[0], dev[1], dev[2], pw, dev[3], want_grad=False)
    assert none is None and torch.equal(only, loss)
    # in place, and inside a wider buffer whose other elements stay
    wide = torch.full((N, M + 3), 5.0, dtype=DT[dtype], device=DEV)
    wide[:, 1:M + 1] = dev[0]
    again, same = D.router_loss(wide[:, 1:M + 1], dev[1], dev[2], pw, dev[3], out=wide[:, 1:M + 1])
    assert torch.equal(again, loss) and torch.equal(wide[:, 1:M + 1], grad)
    assert (wide[:, 0] == 5.0).all() and (wide[:, M + 1:] == 5.0).all()
    for r in sorted({0, 1 % N, 2 % N, N - 1}):
        w = float(weights[r])
        lab = np.zeros(M, dtype=bool)
        lab[[int(of[i]) for i in ids[r].tolist() if 0 <= i < V]] = True
        s = f64(scores[r])
        cost, d = O.router_row(s, lab, float(np.float32(pw)))
        rel = (1.5 * np.abs(s) + 16) * U
        if w == 0.0:
            assert float(loss[r]) == 0.0 and not grad[r].any()
            continue
        assert abs(float(loss[r]) - cost.sum()) <= (cost * rel).sum() + cost.sum() * U + 1e-37
        tol = w * np.abs(d) * (rel + torch.finfo(DT[dtype]).eps / 2) + 1e-37
        assert (np.abs(f64(grad[r]) - w * d) <= tol).all()


def test_router_gradient_against_differences():
    V, M = 500, 30
    g = torch.Generator().manual_seed(3)
    s = torch.randn((1, M), generator=g)
    of = torch.randint(0, M, (V,), generator=g, dtype=torch.int32).to(DEV)
    ids = torch.randint(0, V, (1, 6), generator=g, dtype=torch.int32).to(DEV)
    _, grad = D.router_loss(s.to(DEV), ids, of, 4.0)
    h = 2.0 ** -5
    for m in range(M):
        two = s.repeat(2, 1)
        two[0, m] += h
        two[1, m] -= h
        loss, _ = D.router_loss(two.to(DEV), ids.repeat(2, 1), of, 4.0, want_grad=False)
        # the loss (about 30) is rounded to 2^-20, over 2h = 2^-4; third derivative at most 4 / 8, h^2 / 6 of it
        assert abs((float(loss[0]) - float(loss[1])) / (2 * h) - float(grad[0, m])) <= 2.0 ** -15 + 1e-4


def test_router_infinite_scores():
    of = torch.arange(8, dtype=torch.int32, device=DEV)
    s = torch.zeros((3, 8), device=DEV)
    s[0, 3], s[0, 5] = -math.inf, math.inf
    s[1, 3] = math.inf
    s[2, 0] = math.nan
    ids = torch.tensor([[1, -1], [3, 3], [2, -1]], dtype=torch.int32, device=DEV)
    loss, grad = D.router_loss(s, ids, of)
    assert float(loss[0]) == math.inf and abs(float(loss[1]) - 7 * math.log(2)) < 1e-5 and math.isnan(float(loss[2]))
    assert float(grad[0, 3]) == 0.0 and float(grad[0, 5]) == 1.0 and float(grad[1, 3]) == 0.0


def test_learning_graph_replays_agree_with_eager():
    N, V, K, M = 5, 3000, 6, 40
    logits, ids, values = (x.to(DEV) for x in problem(N, V, K, "bf16", 20))
    of = torch.randint(0, M, (V,), dtype=torch.int32, device=DEV)
    scores = torch.randn((N, M), device=DEV)
    ws = D.distill_workspace(N, V)
    out, rout = torch.empty_like(logits), torch.empty_like(scores)
    for _ in range(2):
        D.distill(logits, ids, values, tail=True, out=out, ws=ws)
        D.router_loss(scores, ids, of, out=rout)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, stats, _ = D.distill(logits, ids, values, tail=True, want_stats=True, out=out, ws=ws)
        rloss, _ = D.router_loss(scores, ids, of, out=rout)
    for seed in range(4):
        a, b, c = problem(N, V, K, "bf16", 30 + seed)
        logits.copy_(a)
        ids.copy_(b)
        values.copy_(c)
        scores.normal_()
        want = D.distill(logits, ids, values, tail=True, want_stats=True)
        rwant = D.router_loss(scores, ids, of)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((loss, stats, out, rloss, rout), (*want, *rwant)):
            assert torch.equal(x, y)


def test_learning_refusals():
    N, V, K = 3, 50, 2
    z = torch.zeros((N, V), device=DEV)
    ids = torch.zeros((N, K), dtype=torch.int32, device=DEV)
    val = torch.zeros((N, K), device=DEV)
    for bad in (lambda: D.distill(z.cpu(), ids, val), lambda: D.distill(z, ids[:2], val[:2]),
                lambda: D.distill(z, ids, val[:, :1]), lambda: D.distill(z.t(), ids, val),
                lambda: D.distill(z, ids, val, out=torch.zeros((N, V + 1), device=DEV)),
                lambda: D.distill(z, ids, val, weights=torch.ones(N - 1, device=DEV)),
                lambda: D.router_loss(z, ids[:1], ids.view(-1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: D.distill(z.double(), ids, val), lambda: D.distill(z, ids.long(), val),
                lambda: D.router_loss(z, ids, ids.view(-1).long())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: D.distill(z, ids, val, temperature=0.0), lambda: D.distill(z, ids, val, out=z),
                lambda: D.router_loss(z, ids, ids.view(-1), pos_weight=0.0)):
        with pytest.raises(D.DynaError) as err:
            bad()
        assert err.value.status == D.ERR_INVALID_ARG
    with pytest.raises(D.DynaError) as err:
        D.distill(z, ids, val, ws=torch.empty(1, dtype=torch.uint8, device=DEV))
    assert err.value.status == D.ERR_WORKSPACE
    empty = D.distill(z[:0], ids[:0], val[:0])
    assert empty[0].numel() == 0 and empty[2].shape == (0, V)


@pytest.mark.parametrize("N,dtype,K", [(2, "f32", 1024), (65, "bf16", 200), (1030, "bf16", 7)])
def test_distill_over_the_largest_vocabulary(N, dtype, K):
    """Parts of every length, up to 65536 entries with a bit for each."""
    V = 1 << 20
    logits, ids, values = problem(2, V, K, dtype, 3)
    pick = torch.arange(N) % 2
    z = logits.to(DEV)[pick.to(DEV)]
    dev = [x[pick].to(DEV) for x in (ids, values)]
    loss, stats, grad = D.distill(z, *dev, 1.0, True, want_stats=True)
    back = D.distill_grad(z, stats, *dev, 1.0, True)
    for r in (0, N - 1):
        one = [x[r:r + 1].cpu() for x in (z, *dev)]
        check_rows(*one, 1.0, True, None, loss[r:r + 1], stats[r:r + 1], grad[r:r + 1])
        check_rows(*one, 1.0, True, None, None, None, back[r:r + 1])
    assert torch.equal(loss, loss[pick.to(DEV)]) and torch.equal(grad[N - 1], grad[(N - 1) % 2])


@pytest.mark.parametrize("N", [5, 170])
@pytest.mark.parametrize("value", [800.0, 1e10, 1e30, 3e38])
def test_values_that_are_no_log_probabilities_show(N, value):
    """exp(value) is above every number: such a row's loss is not finite, by either
    kernel, and the rows beside it keep theirs."""
    V, K = 3000, 8
    logits, ids, values = problem(5, V, K, "f32", 33)
    pick = torch.arange(N) % 5
    logits, ids, values = logits[pick], ids[pick], values[pick]
    values[1, 3] = value
    dev = [x.to(DEV) for x in (logits, ids, values)]
    loss, _, grad = D.distill(*dev, 1.0, True)
    only, _, _ = D.distill(*dev, 1.0, True, want_grad=False)
    assert not math.isfinite(float(loss[1])) and not math.isfinite(float(only[1]))
    check_rows(logits, ids, values, 1.0, True, None, loss, None, grad, [0, 2, 3, 4])
