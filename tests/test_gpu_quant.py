"""Four-bit rows on the GPU: quantisation, products and the gathered head against the fp64 oracle.

Quantisation is compared exactly.  A product's terms are exact, and a term takes part in at most n roundings of its sum
(n = columns + 64 here, three times the columns for fp32 contexts: one for every column that can be added one after the
other, and the joins of the waves' sums), so it is within n 2^-24 of the sum of the terms' magnitudes; a bf16 result
in addition within 2^-8 of itself.  Products of small whole numbers are exact.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import quant_oracle as O
from paper_2510_13847_amd import dynahead as D

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def framed(shape, dtype, pad=(0, 0), fill=float("nan")):
    """A tensor of this shape inside a larger one: pad[0] elements in front, pad[1] between rows."""
    rows, cols = shape
    base = torch.full((pad[0] + max(rows, 1) * (cols + pad[1]) + 8,), fill, dtype=dtype, device="cuda")
    return base[pad[0]:].as_strided((rows, cols), (cols + pad[1], 1)), base


def on_gpu(x, pad=(0, 0)):
    t, _ = framed(x.shape, x.dtype, pad, 0.0)
    t.copy_(x)
    return t


def rows_of(kind, n, d, dtype, seed):
    g = gen(seed)
    x = torch.randn((n, d), generator=g)
    if kind == "spread":  # blocks of every magnitude
        x *= torch.exp2(torch.randint(-60, 60, (n, -(-d // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :d]
    elif kind == "ends":  # the ends of the exponents, zeros of both signs, whole blocks of zeros
        x *= torch.exp2(torch.randint(-149, 127, (n, -(-d // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :d]
        x[torch.rand((n, d), generator=g) < 0.2] = 0.0
        x[torch.rand((n, d), generator=g) < 0.1] = -0.0
        x[:, :32] = 0.0
    elif kind == "ties":  # halfway between neighbours, and next to it
        x = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 4.0])[torch.randint(0, 9, (n, d), generator=g)]
        x *= 1.0 + (torch.randint(-1, 2, (n, d), generator=g).float() * 2.0 ** (-7 if dtype == "bf16" else -23))
        x[:, ::32] = 4.0
    elif kind == "bad":
        x[0, 0] = float("inf")
        x[n // 2, d // 2] = float("nan")
        x[n - 1, d - 1] = -float("inf")
    return x.to(DT[dtype])


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,pad", [(1, 1, (0, 0)), (1, 31, (1, 0)), (15, 32, (0, 3)), (16, 33, (3, 1)), (17, 128, (0, 0)),
                                     (33, 129, (1, 7)), (5, 511, (5, 1)), (16, 512, (0, 0)), (31, 513, (0, 1)),
                                     (40, 1000, (2, 6)), (3, 5376, (0, 0)), (2, 8192, (1, 1))])
def test_rows_and_back(n, d, pad, dtype):
    x = rows_of("plain", n, d, dtype, n * 10007 + d)
    q = D.quantize_rows(on_gpu(x, pad))
    want = torch.tensor(O.quantized_rows(x.double().numpy()))
    for out_type in DT.values():
        out, base = framed((n, d), out_type, pad)
        D.dequantize_rows(q, out=out)
        assert torch.equal(out.cpu().double(), want)
        # nothing else of the frame was written
        assert int(torch.isnan(base).sum()) == base.numel() - n * d
        assert torch.equal(D.dequantize_rows(q, dtype=out_type).cpu().double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["spread", "ends", "ties", "bad"])
def test_values_at_the_edges(kind, dtype):
    x = rows_of(kind, 21, 200, dtype, 5)
    want = torch.tensor(O.quantized_rows(x.double().numpy()))
    got = D.dequantize_rows(D.quantize_rows(x.cuda())).cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def test_padding_holds_zeros_and_quantising_again_changes_nothing():
    x = rows_of("plain", 19, 300, "f32", 8).cuda()
    q = D.quantize_rows(x)
    wide = torch.zeros((32, 384), device="cuda")
    wide[:19, :300] = x
    assert torch.equal(D.quantize_rows(wide).data, q.data)
    values = D.dequantize_rows(q)
    assert torch.equal(D.dequantize_rows(D.quantize_rows(values)), values)
    # written again, over what another matrix left
    again = D.quantize_rows(rows_of("bad", 19, 300, "f32", 9).cuda())
    assert D.quantize_rows(x, out=again) is again and torch.equal(again.data, q.data)


def test_many_rows():
    """Past 2^31 elements: row offsets in 64 bits."""
    n, d = 270000, 8192
    x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    q = D.quantize_rows(x)
    back = D.dequantize_rows(q, dtype=torch.bfloat16)
    for r in (0, 131071, 262143, 262144, 262145, n - 1):
        want = O.quantized_rows(x[r:r + 1].double().cpu().numpy())
        assert torch.equal(back[r].cpu().double(), torch.tensor(want[0])), r


# ---------------------------------------------------------------- products
def whole(n, d, seed, power=0):
    """Rows that four bits hold: whole numbers of halves."""
    g = gen(seed)
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])[torch.randint(0, 8, (n, d), generator=g)]
    return v * (1 - 2 * torch.randint(0, 2, (n, d), generator=g)) * 2.0 ** power


def scaled_whole(n, d, seed):
    """The same with another power of two in each block."""
    x = whole(n, d, seed)
    x[:, ::32] = 4.0  # fixes each block's scale
    return x * torch.exp2(torch.randint(-2, 3, (n, -(-d // 32)), generator=gen(seed + 1)).float()).repeat_interleave(32, 1)[:, :d]


def contexts(kind, B, d, seed, pad=(0, 0)):
    """Whole numbers in the type, as the call takes them and in float64."""
    if kind == "four":
        x = whole(B, d, seed)
        x[:, ::32] = 6.0
        return D.quantize_rows(x.cuda()), x.double()
    x = torch.randint(-9, 10, (B, d), generator=gen(seed)).to(DT[kind])
    return on_gpu(x, pad), x.double()


SHAPES = [(1, 1, 1), (1, 16, 128), (2, 15, 33), (4, 8192, 256), (5, 100, 640), (6, 17, 1000), (1, 1000, 4096),
          (13, 333, 2000), (16, 50, 512), (17, 129, 513), (16, 40, 4100), (33, 300, 200), (40, 65, 5376), (64, 257, 128),
          (65, 20, 8192), (100, 31, 96), (128, 500, 384), (130, 700, 1536), (257, 513, 640), (300, 1100, 130)]


@pytest.mark.parametrize("kind", ["bf16", "f32", "four"])
@pytest.mark.parametrize("B,n,d", SHAPES)
def test_whole_numbers_are_exact(B, n, d, kind):
    W = scaled_whole(n, d, 3 * n + d)
    q = D.quantize_rows(W.cuda())
    assert torch.equal(D.dequantize_rows(q).cpu(), W)
    a, exact = contexts(kind, B, d, B, (1, 3))
    # |sum| <= 54 * 24 * 8192 / 2^-3 units < 2^24: no rounding anywhere
    want = exact @ W.double().t()
    out, base = framed((B, n), torch.float32, (3, 5))
    assert D.quant_product(a, q, out=out) is out
    assert torch.equal(out.cpu().double(), want)
    assert int(torch.isnan(base).sum()) == base.numel() - B * n


# tables of rows long enough for the large tiles: of 32, 64, 128 and 256 contexts by 256 rows, ends inside a tile and
# inside every place of a unit of four steps
TALL = [(20, 66000, 130), (31, 65537, 384), (33, 65600, 513), (64, 65537, 256), (65, 66001, 640), (128, 65600, 96),
        (129, 33000, 385), (200, 33100, 700), (257, 33000, 1000), (300, 65793, 60),
        (256, 65600, 200), (500, 33000, 385), (90, 17000, 300), (17, 30000, 1000)]


@pytest.mark.parametrize("kind", ["bf16", "f32", "four"])
@pytest.mark.parametrize("B,n,d", TALL)
def test_whole_numbers_are_exact_over_tall_tables(B, n, d, kind):
    W = scaled_whole(n, d, n + d)
    a, exact = contexts(kind, B, d, B, (1, 3))
    # |terms| <= 54 * 24 in units of 2^-4: no rounding in 64 bits or in 32
    want = (exact.cuda() @ W.double().cuda().t().contiguous()).float()
    q = D.quantize_rows(W.cuda())
    assert torch.equal(D.quant_product(a, q), want)
    out, base = framed((B, n), torch.bfloat16, (3, 5))
    D.quant_product(a, q, out=out)
    assert torch.equal(out, want.to(torch.bfloat16))
    assert int(torch.isnan(base).sum()) == base.numel() - B * n


@pytest.mark.parametrize("B,n,d", [(1, 40, 300), (3, 100, 4096), (16, 37, 1000), (70, 200, 520), (150, 300, 256)])
def test_fp32_contexts_keep_all_their_bits(B, n, d):
    """One column of every row is not zero: the product is the context's value times it, exactly."""
    g = gen(B)
    at = torch.randint(0, d, (n,), generator=g)
    W = torch.zeros((n, d))
    W[torch.arange(n), at] = torch.tensor([1.0, -2.0, 0.5, 4.0])[torch.randint(0, 4, (n,), generator=g)]
    a = torch.randn((B, d), generator=g) * torch.exp2(torch.randint(-30, 30, (B, d), generator=g).float())
    out = D.quant_product(a.cuda(), D.quantize_rows(W.cuda()))
    assert torch.equal(out.cpu(), a[:, at] * W[torch.arange(n), at])


@pytest.mark.parametrize("out_type", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["bf16", "f32", "four"])
@pytest.mark.parametrize("B,n,d", [(1, 300, 4096), (4, 100, 8192), (15, 64, 3584), (48, 200, 1111), (200, 400, 900)])
def test_products(B, n, d, kind, out_type):
    g = gen(d + B)
    W = D.quantize_rows((torch.randn((n, d), generator=g) / d ** 0.5).cuda())
    a = torch.randn((B, d), generator=g) * torch.exp(0.5 * torch.randn(d, generator=g))
    a = D.quantize_rows(a.cuda()) if kind == "four" else a.to(DT[kind]).cuda()
    values = [(D.dequantize_rows(t) if isinstance(t, D.QuantRows) else t).double().cpu().numpy() for t in (a, W)]
    want, size = O.product(*values), O.product_sizes(*values)
    got = D.quant_product(a, W, out_dtype=DT[out_type]).double().cpu().numpy()
    bound = ((3 * d if kind == "f32" else d) + 64) * 2.0 ** -24 * size
    if out_type == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    assert (np.abs(got - want) <= bound).all(), np.abs((got - want) / bound).max()
    assert np.array_equal(got, D.quant_product(a, W, out_dtype=DT[out_type]).double().cpu().numpy())  # run to run


@pytest.mark.parametrize("kind", ["bf16", "f32", "four"])
@pytest.mark.parametrize("B", [1, 20, 140])
def test_static_prefix_and_empty_batch(B, kind):
    q = D.quantize_rows(scaled_whole(300, 200, 4).cuda())
    a, _ = contexts(kind, B, 200, 5)
    every = D.quant_product(a, q)
    for n in (1, 16, 31, 255, 300):
        assert torch.equal(D.quant_product(a, q, n_rows=n), every[:, :n])
    if kind != "four":
        assert D.quant_product(a[:0], q).shape == (0, 300)


@pytest.mark.parametrize("B", [2, 40, 150])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_undefined_values_stay_in_their_row_and_context(B, kind):
    W = scaled_whole(100, 260, 6)
    W[37, 100] = float("nan")
    q = D.quantize_rows(W.cuda())
    a, exact = contexts(kind, B, 260, 7)
    a[1, 259] = float("nan")
    out = D.quant_product(a, q).cpu()
    bad = torch.zeros((B, 100), dtype=torch.bool)
    bad[1], bad[:, 37] = True, True
    assert torch.equal(torch.isnan(out), bad)
    W[37] = 0.0
    assert torch.equal(out[~bad].double(), (exact.nan_to_num(0.0) @ W.double().t())[~bad])
    # an infinite context: infinite where the weight is not zero
    a[1, 259] = float("inf")
    out = D.quant_product(a, q).cpu()[1]
    w = W[:, 259]
    for r in range(100):
        if r != 37:
            assert torch.isnan(out[r]) if w[r] == 0 else out[r] == float("inf") * w[r]


@pytest.mark.parametrize("B", [3, 40, 200])
@pytest.mark.parametrize("n", [100, 33100])
def test_undefined_blocks_of_four_bit_contexts(B, n):
    W = scaled_whole(n, 260, 6)
    W[37, 100] = float("nan")
    x = whole(B, 260, 7)
    x[:, ::32] = 6.0
    exact = x.double().cuda()
    x[1, 259] = float("inf")
    out = D.quant_product(D.quantize_rows(x.cuda()), D.quantize_rows(W.cuda()))
    bad = torch.zeros((B, n), dtype=torch.bool, device="cuda")
    bad[1], bad[:, 37] = True, True
    W[37] = 0.0
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad].double(), (exact @ W.double().cuda().t().contiguous())[~bad])


def test_large_values_of_fp32_contexts():
    """Next to the type's largest number no term of a context overflows."""
    big = float(np.finfo(np.float32).max)
    a = torch.tensor([[big, 0.0], [-big, 1.0]]).cuda()
    out = D.quant_product(a, D.quantize_rows(torch.tensor([[1.0, 0.0], [0.5, 0.0]]).cuda())).cpu()
    assert out.tolist() == [[big, big / 2], [-big, -big / 2]]


# ---------------------------------------------------------------- gathered head
def partition(V, M, seed, empty=True):
    g = gen(seed)
    of = torch.randint(0, M, (V,), generator=g)
    if empty:
        of[of == M // 2] = 0  # an empty cluster
    return of.to(torch.int32)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,V,d,M,k", [(1, 500, 64, 16, 4), (1, 300, 4096, 8, 8), (3, 400, 136, 40, 7), (7, 999, 520, 64, 5),
                                       (16, 640, 1000, 10, 10), (21, 300, 2048, 12, 3), (64, 700, 4104, 30, 6),
                                       (130, 900, 200, 9, 4), (40, 200, 5376, 100, 50), (5, 333, 8192, 7, 2)])
def test_shortlist_logits(B, V, d, M, k, kind):
    layout = D.build_layout(partition(V, M, B).cuda(), scaled_whole(V, d, V).cuda(), M)
    W = D.quantize_rows(layout.W_perm)
    h, exact = contexts(kind, B, d, d)
    clusters = torch.stack([torch.randperm(M, generator=gen(b))[:k] for b in range(B)]).to(torch.int32)
    sel, off, length, ids = D.shortlist(layout, clusters.cuda())
    cap = layout.cap(k) + 3
    out, base = framed((B, cap), torch.float32)
    out.fill_(float("nan"))
    D.quant_shortlist_logits(layout, W, h.contiguous(), sel, off, length, out=out)
    head = layout.W_perm.double().cpu()
    perm = layout.perm.cpu().long()
    token_values = torch.empty_like(head)
    token_values[perm] = head
    for b in range(B):
        n = int(length[b])
        want = exact[b] @ token_values[ids[b, :n].cpu().long()].t()
        assert torch.equal(out[b, :n].cpu().double(), want)
        assert torch.isnan(out[b, n:]).all()


def test_shortlist_logits_against_the_head_it_stands_for():
    """The same calls over the bf16 head of the four-bit rows' values give the same logits."""
    V, d, M, B, k = 3000, 1024, 50, 12, 6
    layout = D.build_layout(partition(V, M, 1).cuda(), scaled_whole(V, d, 2).to(torch.bfloat16).cuda(), M)
    W = D.quantize_rows(layout.W_perm)
    h, _ = contexts("bf16", B, d, 3)
    sel = D.shortlist(layout, torch.stack([torch.randperm(M, generator=gen(b))[:k] for b in range(B)]).int().cuda())
    a = D.shortlist_logits(layout, h, *sel[:3])
    b = D.quant_shortlist_logits(layout, W, h, *sel[:3])
    assert torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0)) and torch.equal(torch.isnan(a), torch.isnan(b))


def test_shortlists_that_repeat_or_miss_clusters():
    V, d, M = 400, 96, 20
    layout = D.build_layout(partition(V, M, 5).cuda(), scaled_whole(V, d, 6).cuda(), M)
    W = D.quantize_rows(layout.W_perm)
    h, _ = contexts("bf16", 3, d, 7)
    clusters = torch.tensor([[10, 10, 10, 10], [-1, 25, 3, 3], [10, 10, -7, 99]], dtype=torch.int32).cuda()
    sel, off, length, ids = D.shortlist(layout, clusters)
    out = D.quant_shortlist_logits(layout, W, h, sel, off, length)
    for b in range(3):
        n = int(length[b])
        assert torch.isnan(out[b, n:]).all() and not torch.isnan(out[b, :n]).any()
    assert int(length[1]) > 0


# ---------------------------------------------------------------- streams and graphs
@pytest.mark.parametrize("B", [3, 40, 150])
def test_another_stream(B):
    W = scaled_whole(500, 640, 1).cuda()
    a, exact = contexts("bf16", B, 640, 2)
    want = (exact @ W.double().cpu().t())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q = D.quantize_rows(W, stream=s)
    out = D.quant_product(a, q, stream=s)
    back = D.dequantize_rows(q, stream=s)
    s.synchronize()
    assert torch.equal(out.cpu().double(), want) and torch.equal(back, W)


@pytest.mark.parametrize("B", [2, 40, 150])
@pytest.mark.parametrize("kind", ["bf16", "four"])
def test_captured_and_replayed(B, kind):
    """A captured quantisation and product, replayed on new inputs, with eager calls of the same between."""
    q = D.quantize_rows(scaled_whole(700, 512, 1).cuda())
    x = whole(B, 512, 2).to(torch.bfloat16).cuda()
    out = torch.empty((B, 700), device="cuda")
    ws = D.quant_product_workspace(B, 512)
    a4 = D.quantize_rows(x)

    def call():
        D.quant_product(D.quantize_rows(x, out=a4) if kind == "four" else x, q, out=out, ws=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3, 7):
        x.copy_(whole(B, 512, seed))
        out.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        assert torch.equal(got, out)
        assert not (got == -1.0).all()


def test_binding_refuses():
    x = torch.zeros((4, 64), device="cuda")
    q = D.quantize_rows(x)
    with pytest.raises(TypeError):
        D.quantize_rows(x.double())
    with pytest.raises(ValueError):
        D.quantize_rows(x.t())
    with pytest.raises(ValueError):
        D.quantize_rows(x[:3], out=q)
    with pytest.raises(ValueError):
        D.quantize_rows(torch.zeros((2, 8193), device="cuda"))
    with pytest.raises(ValueError):
        D.quantize_rows(x[:0])
    for data in (q.data[:-1], q.data.cpu().float(), torch.zeros(2 * q.data.numel(), dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            D.QuantRows(4, 64, data)
    with pytest.raises(ValueError):
        D.dequantize_rows(D.QuantRows(4, 64, q.data.cpu()))
    with pytest.raises(ValueError):
        D.dequantize_rows(q, out=torch.zeros((4, 63), device="cuda"))
    with pytest.raises(ValueError):
        D.quant_product(torch.zeros((2, 65), device="cuda"), q)
    with pytest.raises(ValueError):
        D.quant_product(x, q, out=torch.zeros((4, 5), device="cuda"))
    with pytest.raises(D.DynaError):
        D.quant_product(x, q, n_rows=5)
    with pytest.raises(D.DynaError):
        D.quant_product(x, q, ws=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(D.DynaError):
        D.quant_product(x, q, out=x[:, :4])
