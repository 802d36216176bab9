"""Four-bit rows where their numbers end: every power of two, products of rows and contexts whose powers lie far apart,
and the gathered head's logits of selections that repeat, miss or leave out clusters."""
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


def halves(n, d, seed):
    """e2m1 values, each block with a 4 or a 6."""
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
    x = v[torch.randint(0, 8, (n, d), generator=gen(seed))] * (1 - 2 * torch.randint(0, 2, (n, d), generator=gen(seed + 1)))
    x[:, ::32] = v[6 + torch.randint(0, 2, (n, -(-d // 32)), generator=gen(seed + 2))]
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_block_of_every_power(dtype):
    """Largest magnitudes from the type's smallest number to its largest power of two, one block each, with zeros of both
    signs, values that round to zero, ties and both signs of everything."""
    lowest = -133 if dtype == "bf16" else -149
    shape = torch.tensor([1.0, -1.75, 1.25, -0.0, 0.0, 0.0625, -0.0625, 0.1875, -0.3125, 0.875, -0.625, 1.5, 0.03, -0.03,
                          0.4375, -1.125] * 2, dtype=torch.float64)
    x = torch.stack([shape * 2.0 ** e for e in range(lowest, 128)]).to(DT[dtype])  # rounded once
    assert torch.isfinite(x).all() and int((x.abs().amax(1) > 0).sum()) == x.shape[0]
    want = torch.tensor(O.quantized_rows(x.double().numpy()))
    for out_type in DT.values():
        got = D.dequantize_rows(D.quantize_rows(x.cuda()), dtype=out_type).cpu().double()
        assert torch.equal(got, want)
        assert torch.equal(torch.signbit(got), torch.signbit(want))


@pytest.mark.parametrize("kind", ["bf16", "f32", "four"])
@pytest.mark.parametrize("low,high", [(-127, 100), (-126, 120), (-120, 90), (120, -100)])
@pytest.mark.parametrize("B,n,d", [(1, 40, 300), (4, 64, 4096), (16, 40, 640), (40, 130, 520), (64, 65537, 256),
                                   (200, 33100, 96)])
def test_products_of_powers_far_apart(B, n, d, low, high, kind):
    """Whole numbers of halves over 2^low times whole numbers over 2^high: sums of whole numbers below 2^24 in units of
    2^(low + high - 2), so nothing is rounded.  Rows' values are down to 2^-128, numbers below the types' smallest
    normal one."""
    W = halves(n, d, 3)
    q = D.quantize_rows((W * 2.0 ** low).float().cuda())
    assert torch.equal(D.dequantize_rows(q, dtype=torch.bfloat16).double().cpu(), W * 2.0 ** low)
    if kind == "four":
        x = halves(B, d, 9)
        a = D.quantize_rows((x * 2.0 ** high).float().cuda())
    else:
        x = torch.randint(-9, 10, (B, d), generator=gen(5)).double()
        a = (x * 2.0 ** high).to(DT[kind]).cuda()
    want = (x.cuda() @ W.t().contiguous().cuda()) * 2.0 ** (low + high)
    assert torch.equal(D.quant_product(a, q).double(), want)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("low,high", [(-127, 100), (120, -100)])
@pytest.mark.parametrize("B,d", [(1, 64), (7, 1536), (20, 4096)])
def test_gathered_products_of_powers_far_apart(B, d, low, high, kind):
    V, M, k = 500, 16, 5
    of = torch.randint(0, M, (V,), generator=gen(1)).to(torch.int32)
    W = halves(V, d, 3)
    layout = D.build_layout(of.cuda(), (W * 2.0 ** low).float().cuda(), M)
    x = torch.randint(-9, 10, (B, d), generator=gen(5)).double()
    clusters = torch.stack([torch.randperm(M, generator=gen(b))[:k] for b in range(B)]).to(torch.int32)
    sel, off, length, ids = D.shortlist(layout, clusters.cuda())
    z = D.quant_shortlist_logits(layout, D.quantize_rows(layout.W_perm), (x * 2.0 ** high).to(DT[kind]).cuda(), sel, off,
                                 length).double().cpu()
    for b in range(B):
        m = int(length[b])
        assert torch.equal(z[b, :m], x[b] @ W[ids[b, :m].cpu().long()].t() * 2.0 ** (low + high))


@pytest.mark.parametrize("B", [1, 5, 40])
def test_small_fp32_contexts(B):
    """From 2^-110 on three bf16 terms hold all 24 bits; below, the last one ends at 2^-133, so the value is taken to
    2^-134.  One column of a row is not zero."""
    d, n = 300, 50
    at = torch.randint(0, d, (n,), generator=gen(1))
    W = torch.zeros((n, d), dtype=torch.float64)
    W[torch.arange(n), at] = 2.0 ** 60
    q = D.quantize_rows(W.float().cuda())
    for low, high, tol in ((-110, -80, 0.0), (-149, -111, 2.0 ** (60 - 134))):
        a = torch.randn((B, d), generator=gen(2)).clamp(-1.99, 1.99)
        a = torch.where(a.abs() < 1.0, torch.copysign(1.0 + a.abs(), a), a)  # magnitudes in [1, 2)
        a = (a.double() * torch.exp2(torch.randint(low, high, (B, d), generator=gen(3)).double())).float()
        got = D.quant_product(a.cuda(), q).double().cpu()
        assert ((got - a.double()[:, at] * 2.0 ** 60).abs() <= tol).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_logits_of_selections_that_repeat_or_miss_clusters(kind):
    V, d, M = 400, 96, 20
    of = torch.randint(0, M, (V,), generator=gen(5))
    of[of == 10] = 0  # an empty cluster
    W = halves(V, d, 6)
    layout = D.build_layout(of.to(torch.int32).cuda(), W.float().cuda(), M)
    x = torch.randint(-9, 10, (5, d), generator=gen(7)).double()
    clusters = torch.tensor([[10, 10, 10, 10], [-1, 25, 3, 3], [10, 10, -7, 99], [3, 3, 3, 3], [7, 19, 0, 7]],
                            dtype=torch.int32).cuda()
    sel, off, length, ids = D.shortlist(layout, clusters)
    z = D.quant_shortlist_logits(layout, D.quantize_rows(layout.W_perm), x.to(DT[kind]).cuda(), sel, off, length)
    size = torch.bincount(of, minlength=M)
    for b, chosen in enumerate(([], [3], [], [3], [0, 7, 19])):
        names = torch.cat([(of == m).nonzero()[:, 0] for m in chosen]) if chosen else torch.zeros(0, dtype=torch.long)
        assert int(length[b]) == int(size[chosen].sum()) and torch.equal(ids[b, :int(length[b])].cpu().long(), names)
        assert torch.equal(z[b, :len(names)].double().cpu(), x[b] @ W[names].t())
        assert torch.isnan(z[b, len(names):]).all()
