"""Layouts without their 16- or 32-bit rows: entry points that never read W_perm take NULL, the others refuse it.
(Each call is refused for another reason, or has nothing to do, behind the layout's checks.)"""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

from paper_2510_13847_amd import dynahead as D

P = 0x100000


def layout(W):
    cap = (ctypes.c_int32 * 11)(*[100 * i for i in range(11)])
    return D._Layout(1000, 64, 10, D.BF16, W, P, P, ctypes.addressof(cap), 100), cap


@pytest.mark.parametrize("W", [None, 0x1001])  # not read, so of any alignment too
def test_entry_points_that_never_read_the_rows(W):
    lib = D.lib()
    L, keep = layout(W)
    L = ctypes.byref(L)
    assert lib.dyna_shortlist(L, P, 0, 3, P, P, P, P, 300, None) == D.OK
    assert lib.dyna_draft_select(L, P, P, P, P, 0, 3, 300, D.SEL_ARGMAX, 1, 1.0, 0.0, None, P, P, None, None, P, 1 << 30,
                                 None) == D.OK
    quant = ctypes.byref(D._Quant(1000, 64, P))
    assert lib.dyna_quant_shortlist_logits(L, quant, P, D.BF16, 0, 3, P, P, P, P, 300, P, 1 << 30, None) == D.OK
    assert lib.dyna_quant_shortlist_logits(L, quant, P, D.BF16, 2, 3, P, P, P, P, 300, P, 16, None) == D.ERR_WORKSPACE
    assert lib.dyna_token_rows(L, P + 4, None) == D.ERR_INVALID_ARG and b"token_rows" in lib.dyna_last_error()
    rows = ctypes.byref(D._ShortlistRows(ctypes.addressof(L._obj), P, P, P, P, 3, 0))
    assert lib.dyna_token_logprobs(P, D.F32, 100, 100, 4, rows, P, 1, 1.0, 0, P, P, None, None, None, P, 0,
                                   None) == D.ERR_WORKSPACE
    assert lib.dyna_token_logprobs_grad(P, D.F32, 100, 100, 4, rows, P, 1, 1.0, None, P, None, P, 100,
                                        None) == D.ERR_INVALID_ARG and b"stats" in lib.dyna_last_error()
    steps = (D._DraftStep * 1)(D._DraftStep(P, P, P, P, 3, 300, 0, 1.0, 0.0))
    assert lib.dyna_verify_chain(P, D.F32, 1000, 1000, 2000, 2, 1, ctypes.cast(steps, ctypes.c_void_p), None, 1.0, L, P, P,
                                 P, P, P, P, 0, None) == D.ERR_WORKSPACE


@pytest.mark.parametrize("W", [None, 0x1001])
def test_entry_points_that_read_the_rows(W):
    lib = D.lib()
    L, keep = layout(W)
    assert lib.dyna_shortlist_logits(ctypes.byref(L), P, D.BF16, 0, 3, P, P, P, P, 300, P, 1 << 30,
                                     None) == D.ERR_INVALID_ARG
    assert b"layout" in lib.dyna_last_error()


def test_binding():
    of = torch.zeros(16, dtype=torch.int32)
    full = D.Layout(16, 8, 1, torch.zeros((16, 8)), of, of[:2], np.array([0, 16], np.int32), 16)
    assert full._c.wdtype == D.F32 and full._c.W_perm
    less = full.with_weights(None)
    assert less.W_perm is None and not less._c.W_perm and less.perm is of and less.cap(1) == 16
    back = less.with_weights(torch.zeros((16, 8), dtype=torch.bfloat16))
    assert back._c.wdtype == D.BF16 and back._c.W_perm
