"""Best alternatives among equal logits where token ids are large: rows of 2^20 columns, and shortlists over layouts of
more tokens than a row may have columns, on both sides of 2^21."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as O
from paper_2510_13847_amd import dynahead as D

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.mark.parametrize("first", [(1 << 20) - 70000, (1 << 20) - 64, (1 << 20) - 5, (1 << 19) - 30])
@pytest.mark.parametrize("N", [2, 1030])  # rows in parts, and of one workgroup each
def test_equal_logits_near_the_end_of_long_rows(N, first):
    """Weights are 1 and e^-4: off by three roundings of y = 4 log2(e), two steps of 2^-23, their sums' 2^-21 and the
    result's half step."""
    V = 1 << 20
    z = torch.full((N, V), -4.0, dtype=torch.bfloat16, device="cuda")
    z[:, first:] = 0.0
    t = torch.tensor([[V - 1]], dtype=torch.int32).expand(N, 1).contiguous().cuda()
    got = D.token_logprobs(z, t, top=64)
    many = min(V - first, 64)
    ids = list(range(first, first + many)) + list(range(64 - many))
    logp = -math.log((V - first) + first * math.exp(-4.0))
    want = torch.tensor([logp] * many + [logp - 4.0] * (64 - many), dtype=torch.float64)
    assert (got.top_ids.cpu() == torch.tensor(ids, dtype=torch.int32)).all()
    tol = 3 * 5.8 * EPS + 2.0 ** -22 + 2.0 ** -21
    assert ((got.top_logprobs.cpu().double() - want).abs() <= tol + EPS * want.abs()).all()
    assert (got.logprobs.cpu().double() - logp).abs().max() <= tol + EPS * abs(logp)


def test_a_long_row_of_steps_against_the_oracle():
    V = 1 << 20
    z = (torch.arange(V) >> 10).float()[None] / 64.0
    got = D.token_logprobs(z.cuda(), torch.tensor([[V - 1, 0]], dtype=torch.int32).cuda(), top=64)
    given, _, best, _ = O.token_logprobs(z[0].double().numpy(), range(V), [V - 1, 0], 1.0, 64)
    assert got.top_ids[0].tolist() == [i for i, _ in best]
    # weights of the upper steps, 1/64 apart: y < 40 for all that counts
    assert np.abs(got.logprobs[0].cpu().double().numpy() - given).max() <= 3 * 40 * EPS + 2.0 ** -20


def test_an_id_past_the_bits_of_a_small_vocabulary():
    """Rows whose number of columns is a power of two, one less and one more: every id has its bits searched."""
    for V in (1, 2, 3, 4, 63, 64, 65, 1023, 1024, 1025, 16384, 16385, 32768, 32769):
        z = torch.zeros((1, V), device="cuda")
        top = min(64, V)
        got = D.token_logprobs(z, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), top=top)
        assert got.top_ids[0].tolist() == list(range(top)), V


LARGE = 3 << 20  # tokens: past 2^21, where ids have 22 bits


@pytest.fixture(scope="module")
def large():
    """64 clusters of 49152 tokens: ranges of ids, of which neighbours have changed places in their even ids."""
    t = torch.arange(LARGE, device="cuda")
    of = ((t // (LARGE // 64)) ^ (1 - t % 2)).to(torch.int32)
    return D.build_layout(of, torch.zeros((LARGE, 8), dtype=torch.bfloat16, device="cuda"), 64)


@pytest.mark.parametrize("N", [2, 1030])
@pytest.mark.parametrize("kind", ["equal", "two", "few"])
def test_shortlists_of_a_layout_of_more_than_2_to_21_tokens(large, N, kind):
    # clusters whose tokens lie on both sides of 2^21, and all beyond it
    clusters = torch.tensor([[43, 42], [60, 45]], dtype=torch.int32)
    rows = D.shortlist(large, clusters.cuda())
    sel, off, length, ids = [x.repeat(N // 2, 1) if x.dim() == 2 else x.repeat(N // 2) for x in rows]
    n = 2 * (LARGE // 64)
    assert int(length[0]) == n and int(ids[0, :n].min()) < 1 << 21 < int(ids[0, :n].max()) and int(ids[1, :n].min()) > 1 << 21
    value = {"equal": torch.zeros(n), "two": (torch.arange(n) % 2).float(),
             "few": (torch.arange(n) % 1500 == 7).float()}[kind]  # 66 tokens at the top
    z = torch.full((N, ids.shape[1]), float("nan"), device="cuda")
    z[:, :n] = value.cuda()
    where = D.ShortlistRows(large, sel.contiguous(), off.contiguous(), length.contiguous())
    got = D.token_logprobs(z, ids[:, 5].contiguous(), top=64, rows=where)
    for r in (0, 1):
        names = ids[r, :n].cpu()
        at_top = names[value == value.max()].sort().values[:64]
        assert torch.equal(got.top_ids[r].cpu(), at_top)
        assert torch.equal(got.top_ids[r::2], got.top_ids[r].expand(N // 2, 64))
    total = float(torch.exp(value.double() - value.max()).sum())
    assert (got.top_logprobs.cpu().double() + math.log(total)).abs().max() <= 2.0 ** -20
    assert (got.logprobs.cpu().double() + math.log(total) - float(value[5] - value.max())).abs().max() <= 2.0 ** -20


def test_a_short_row_past_2_to_21(large):
    """One sweep, whose candidates are more than the list keeps."""
    sel, off, length, ids = D.shortlist(large, torch.tensor([[50]], dtype=torch.int32).cuda())
    z = torch.zeros((1, 600), device="cuda")
    got = D.token_logprobs(z, ids[:, 0].contiguous(), top=64, rows=D.ShortlistRows(large, sel, off, length))
    assert torch.equal(got.top_ids[0], ids[0, :600].sort().values[:64])
