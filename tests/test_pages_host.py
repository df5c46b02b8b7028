"""Host side of the operations on chosen pages: what they refuse before anything is launched (the pointers are never followed, so this
runs without a GPU)."""
import ctypes as C

import pytest

from test_paged_host import BAD_CACHES, CAPACITY, INVALID, P, WORKSPACE, _cache, nnc  # noqa: F401


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_caches_that_are_refused(nnc, bad):
    ref = C.byref(_cache(nnc, **bad))
    assert nnc.lib.nnc_op_page_bounds(ref, P, P, P, 1, None) == INVALID
    assert nnc.lib.nnc_op_score_pages(P, ref, P, P, P, 0, 1, 4, 512, None) == INVALID
    assert nnc.lib.nnc_op_attn_selected_paged(P, ref, P, P, P, 3, P, None, 0, 1, 4, 512, 512, 1.0, P, 16 << 20, None) == INVALID


def test_bounds_and_score_calls_that_are_refused_and_empty_ones(nnc):
    ref = C.byref(_cache(nnc))
    good = dict(cache=ref, bounds=P, lens=P, first=None, batch=4)
    call = lambda **kw: nnc.lib.nnc_op_page_bounds(*{**good, **kw}.values(), None)
    for bad in (dict(cache=None), dict(bounds=None), dict(lens=None), dict(bounds=P + 8), dict(lens=P + 2), dict(first=P + 1), dict(batch=-1), dict(batch=5)):
        assert call(**bad) == INVALID, bad
    assert call(batch=0) == 0 and call(batch=0, bounds=None, lens=None) == 0
    assert call(cache=C.byref(_cache(nnc, n_seqs=1 << 20)), batch=1 << 16) == CAPACITY
    good = dict(q=P, cache=ref, bounds=P, lens=P, scores=P, type=1, batch=4, nq=8, qs=1024)
    call = lambda **kw: nnc.lib.nnc_op_score_pages(*{**good, **kw}.values(), None)
    half, codes = C.byref(_cache(nnc, type=2)), C.byref(_cache(nnc, type=3, k_scale=P, v_scale=P))
    for bad in (dict(q=None), dict(cache=None), dict(bounds=None), dict(lens=None), dict(scores=None), dict(type=2), dict(type=3), dict(type=-1),
                dict(cache=half), dict(cache=codes, type=3), dict(batch=-1), dict(batch=5), dict(nq=0), dict(nq=7), dict(q=P + 8), dict(bounds=P + 4),
                dict(qs=1023), dict(type=0, qs=1022), dict(lens=P + 2), dict(scores=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(nq=2 * 129) == CAPACITY and call(batch=0) == 0 and call(batch=0, q=None, bounds=None, scores=None) == 0


def test_selection_calls_that_are_refused_and_empty_ones(nnc):
    good = dict(scores=P, lens=P, pages=P, counts=P, batch=2, heads=2, columns=9, page=16, n=4, first=1, last=1)
    call = lambda **kw: nnc.lib.nnc_op_select_pages(*{**good, **kw}.values(), None)
    for bad in (dict(scores=None), dict(lens=None), dict(pages=None), dict(counts=None), dict(scores=P + 2), dict(pages=P + 1), dict(counts=P + 3), dict(lens=P + 2),
                dict(batch=-1), dict(heads=0), dict(columns=0), dict(page=8), dict(page=48), dict(page=512), dict(n=0), dict(n=-1), dict(first=-1),
                dict(last=-1), dict(first=3, last=2), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
        assert call(**bad) == INVALID, bad
    assert call(batch=1 << 20, heads=1 << 12) == CAPACITY and call(columns=2 ** 31 - 1) == CAPACITY
    for n in (2 ** 30 + 1, 2 ** 31 - 1025):   # indices are 32-bit numbers, with room for a CTA's step behind the last one
        assert call(columns=n) == CAPACITY and call(n=n) == CAPACITY
    assert call(batch=0) == 0 and call(batch=0, scores=None, pages=None) == 0


def test_attention_calls_that_are_refused_and_empty_ones(nnc):
    good = dict(q=P, cache=C.byref(_cache(nnc)), lens=P, pages=P, counts=P, list_len=3, out=P, lse=None, type=1, batch=4, nq=8, qs=1024, os=1024, scale=1.0,
                scratch=P, nbytes=16 << 20)
    call = lambda **kw: nnc.lib.nnc_op_attn_selected_paged(*{**good, **kw}.values(), None)
    codes, half = C.byref(_cache(nnc, type=3, k_scale=P, v_scale=P)), C.byref(_cache(nnc, type=2))
    for bad in (dict(q=None), dict(cache=None), dict(lens=None), dict(pages=None), dict(counts=None), dict(out=None), dict(scratch=None), dict(type=2), dict(type=3),
                dict(cache=half), dict(cache=codes, type=3), dict(batch=-1), dict(batch=5), dict(nq=0), dict(nq=7), dict(list_len=0), dict(list_len=-3),
                dict(q=P + 8), dict(out=P + 8), dict(qs=1023), dict(os=4), dict(type=0, qs=1022), dict(lens=P + 2), dict(pages=P + 2), dict(counts=P + 1), dict(lse=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(nbytes=(16 << 20) - 1) == WORKSPACE and call(scratch=P + 128) == WORKSPACE
    assert call(list_len=1 << 26) == CAPACITY
    assert call(batch=0) == 0 and call(batch=0, q=None, out=None, lens=None, pages=None, scratch=None) == 0


def test_prefix_calls_that_are_refused_and_empty_ones(nnc):
    nbytes = nnc.lib.nnc_attn_prefix_scratch_bytes(4, 8, 128)
    assert nbytes > 16 << 20 and nnc.lib.nnc_attn_prefix_scratch_bytes(0, 8, 128) > 0
    assert [nnc.lib.nnc_attn_prefix_scratch_bytes(*x) for x in ((-1, 8, 128), (4, 0, 128), (4, 8, 96))] == [0, 0, 0]
    good = dict(q=P, cache=C.byref(_cache(nnc)), lens=P, starts=P, shared=P, n_groups=2, out=P, lse=None, type=1, batch=4, nq=8, qs=1024, os=1024, scale=1.0,
                scratch=P, nbytes=nbytes)
    call = lambda **kw: nnc.lib.nnc_op_attn_prefix_paged(*{**good, **kw}.values(), None)
    codes, half = C.byref(_cache(nnc, type=3, k_scale=P, v_scale=P)), C.byref(_cache(nnc, type=2))
    for bad in (dict(q=None), dict(cache=None), dict(lens=None), dict(starts=None), dict(shared=None), dict(out=None), dict(scratch=None), dict(type=2), dict(type=3),
                dict(cache=half), dict(cache=codes, type=3), dict(batch=-1), dict(batch=5), dict(nq=0), dict(nq=7), dict(n_groups=0), dict(n_groups=5), dict(n_groups=-1),
                dict(q=P + 8), dict(out=P + 8), dict(qs=1023), dict(os=4), dict(type=0, qs=1022), dict(lens=P + 2), dict(starts=P + 2), dict(shared=P + 1), dict(lse=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(nbytes=nbytes - 1) == WORKSPACE and call(scratch=P + 128) == WORKSPACE
    assert call(cache=C.byref(_cache(nnc, n_pages=1 << 24))) == CAPACITY
    assert call(batch=0) == 0 and call(batch=0, q=None, out=None, lens=None, starts=None, scratch=None) == 0
