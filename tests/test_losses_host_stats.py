"""Refusals of the token log-probabilities' entries with row statistics, before any device work."""
import ctypes as C

import paper_2203_16340_amd as L
from paper_2203_16340_amd import losses as S


def _lg(**kw):
    a = dict(dtype=1, rows=4, vocab=100, ld=100, z=0x10000, temperature=1.0, grad=0x90000, ld_grad=100)
    a.update(kw)
    return S.Logits(*a.values())


def test_top_goes_with_sum():
    lib, b = L.lib(), C.byref(_lg())
    ws, n = 0x100000, 1 << 30
    for top, total in ((0x4000, None), (None, 0x5000)):
        assert lib.lbfgsb_token_logprob_stats(b, 0x1000, 0x2000, 0x3000, None, None, top, total, ws, n, None) == L.E_INVALID_ARG
    assert lib.lbfgsb_token_logprob_stats(b, None, 0x2000, 0x3000, None, None, 0x4000, 0x5000, ws, n, None) == L.E_INVALID_ARG


def test_the_way_back_needs_both():
    lib, b = L.lib(), C.byref(_lg())
    for args in ((None, 0x2000, 0x3000, None, 0x4000, None), (0x1000, None, 0x3000, None, 0x4000, None), (0x1000, 0x2000, None, None, 0x4000, None),
                 (0x1000, 0x2000, 0x3000, None, None, None), (0x1000, 0x2000, 0x3000, None, 0x4000, 0x5000)):
        assert lib.lbfgsb_token_logprob_stats_grad(b, *args, None) == L.E_INVALID_ARG, args
    bad = C.byref(_lg(grad=None))
    assert lib.lbfgsb_token_logprob_stats_grad(bad, 0x1000, 0x2000, 0x3000, None, 0x4000, None, None) == L.E_INVALID_ARG


def test_no_rows():
    none = C.byref(_lg(rows=0))
    assert L.lib().lbfgsb_token_logprob_stats(none, None, None, None, None, None, None, None, None, 0, None) == L.OK
    assert L.lib().lbfgsb_token_logprob_stats_grad(none, None, None, None, None, None, None, None) == L.OK
