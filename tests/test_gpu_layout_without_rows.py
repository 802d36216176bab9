"""A head kept in four bits alone: drafting, scoring and verification over a layout that holds no 16-bit rows."""
from __future__ import annotations

import pytest
import torch

from paper_2510_13847_amd import dynahead as D

pytestmark = pytest.mark.gpu


def test_a_draft_step_without_the_sixteen_bit_rows():
    V, d, M, k, B = 3000, 256, 50, 6, 5
    g = torch.Generator().manual_seed(1)
    of = torch.randint(0, M, (V,), generator=g).to(torch.int32).cuda()
    full = D.build_layout(of, (torch.randn((V, d), generator=g) / d ** 0.5).to(torch.bfloat16).cuda(), M)
    W = D.quantize_rows(full.W_perm)
    h = torch.randn((B, d), generator=g).to(torch.bfloat16).cuda()
    clusters = torch.stack([torch.randperm(M, generator=g)[:k] for _ in range(B)]).to(torch.int32).cuda()
    target = torch.randn((B, 2, V), generator=g).cuda()
    u, uv, gr = [torch.rand(s, generator=g).cuda() for s in ((B,), (B, 2), (B,))]

    def cycle(layout):
        sel = D.shortlist(layout, clusters)
        z = D.quant_shortlist_logits(layout, W, h, *sel[:3], ws=D.workspace(layout, None, B, k, layout.cap(k)))
        out = D.draft_select(layout, z, *sel[:3], mode=D.SEL_SAMPLE | D.SEL_TOPK, k_t=3, uniforms=u)
        rows = D.ShortlistRows(layout, *sel[:3])
        s = D.token_logprobs(z, out["sample"], top=4, rows=rows, want_stats=True)
        grad = D.token_logprobs_grad(z, s.stats, out["sample"], gr, rows=rows)
        v = D.verify_chain(target, [D.DraftStep(out["sample"], s.logprobs, z, clusters)], uv, layout=layout)
        return sel[3], z.nan_to_num(0.0), out["ids"], s.logprobs, s.entropy, s.top_ids, grad, v.ids, v.lengths

    less = full.with_weights(None)
    for a, b in zip(cycle(less), cycle(full)):
        assert torch.equal(a, b)
    with pytest.raises(D.DynaError):
        sel = D.shortlist(less, clusters)
        D.shortlist_logits(less, h, *sel[:3])
