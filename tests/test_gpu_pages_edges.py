"""Chosen pages where tables and tables' widths are out of the ordinary."""
import pytest
import torch

from test_gpu_paged import BF16, _fill, _gen, _ints, _paged, _randn, nnc, scratch  # noqa: F401
from test_gpu_pages import _check_selected, _lists, _select

pytestmark = pytest.mark.gpu


def test_every_page_that_the_pool_does_not_have_sets_the_status(nnc, scratch):
    lens = [100, 100]
    cache = _paged(nnc, BF16, lens, 16, 2, 64, 6)
    held = _fill(nnc, cache, lens, 1)
    q = _randn(_gen(2), 2, 4, 64, dtype=BF16)
    pages, counts = _lists([[[0, 3, 2], [6, 1, 0]], [[2, 3, 4], [5, 4, 0]]], 3)
    left = [[[0, 2], [6, 1, 0]], [[2, 3, 4], [5, 4, 0]]]
    for bad in (-1, -2, -3, -2 ** 31, cache.n_pages, 2 ** 31 - 1):
        cache.page_table[0, 3] = bad
        out, lse = nnc.op_attn_selected_paged(q, cache, _ints(lens), pages, counts, scratch=scratch, want_lse=True)
        assert nnc.op_status() == 0x100, bad
        _check_selected(out, lse, q, held, lens, left, 16, 0.125, BF16)


@pytest.mark.parametrize("columns", [1024, 1025, 2560, 2561, 4608, 4609, 8192, 8193, 8704, 8705, 40960, 40961])
def test_selection_at_both_ends_of_every_form_s_widths(nnc, columns):
    """Scores of few different values, so that ties decide, for rows that use all of the table, little of it and none."""
    lens = [columns * 16, (columns - 1) * 16 + 1, 40 * 16, 0]
    scores = torch.randint(0, 50, (4, 2, columns), generator=_gen(columns), device="cuda").float()
    scores[1, 1] = -7.5
    for n in (64, 1000):
        pages, counts = nnc.op_select_pages(scores, _ints(lens), 16, n, 2, 1)
        want, want_counts = _select(scores, lens, 16, n, 2, 1)
        assert torch.equal(pages.cpu(), want) and torch.equal(counts.cpu(), want_counts)
