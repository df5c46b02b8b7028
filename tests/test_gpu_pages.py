"""Pages chosen by a score: bounds, scores, selection and the attention over what was selected, against plain 64-bit forms of the same
operations, at the sizes, lists and lengths where they can go wrong.  Bounds of errors as in test_gpu_paged."""
import math

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, F32, TYPES, _check_attention, _fill, _gen, _ints, _paged, _randn, nnc, quantise64, scratch  # noqa: F401

pytestmark = pytest.mark.gpu


def _bounds64(held, lens, page):
    """[lowest, highest] of every page of every sequence: lists of [pages][heads][2][d]."""
    got = []
    for k, n in zip(held[0], lens):
        got.append([torch.stack([k[:, lo:min(n, lo + page)].amin(1), k[:, lo:min(n, lo + page)].amax(1)], 1) for lo in range(0, n, page)])
    return got


# ---- bounds ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv", [BF16, F16, E4M3], ids=str)
@pytest.mark.parametrize("heads,d,page", [(1, 64, 16), (8, 128, 64), (3, 128, 256), (5, 64, 32), (2, 128, 128)])
def test_bounds(nnc, kv, heads, d, page):
    lens = [0, 1, page - 1, page, page + 1, 3 * page + 5, 700]
    cache = _paged(nnc, kv, lens, page, heads, d, heads)     # rows past a length are NaN
    held = _fill(nnc, cache, lens, 3)
    want = _bounds64(held, lens, page)
    bounds = nnc.page_bounds(cache)
    assert bounds.dtype is (F16 if kv is F16 else BF16)
    bounds.fill_(7.0)
    assert nnc.op_page_bounds(cache, bounds, _ints(lens)) is bounds
    seen = torch.zeros(cache.n_pages, dtype=torch.bool, device="cuda")
    for b, pages in enumerate(want):
        for i, x in enumerate(pages):
            at = cache.page_table[b, i].long()
            seen[at] = True
            assert torch.equal(bounds[at].double(), x), (b, i)     # minima and maxima are values of the cache: exact
    assert (bounds[~seen] == 7).all()
    # from a position on: only the pages that hold one of the new positions, and all of their rows
    first = [0, 1, 0, page - 1, page, 2 * page + 1, 699]
    bounds.fill_(7.0)
    nnc.op_page_bounds(cache, bounds, _ints(lens), _ints(first))
    for b, pages in enumerate(want):
        for i, x in enumerate(pages):
            got = bounds[cache.page_table[b, i].long()].double()
            touched = first[b] < lens[b] and i >= first[b] // page
            assert torch.equal(got, x) if touched else (got == 7).all(), (b, i)
    assert nnc.op_status() == 0
    assert nnc.op_page_bounds(cache, bounds, _ints([])) is bounds


def test_bounds_of_numbers_that_are_not_finite_and_of_signed_zeros(nnc):
    for kv in (BF16, F16):
        cache = _paged(nnc, kv, [40], 16, 1, 64, 1)
        x = _randn(_gen(1), 40, 1, 64)
        x[3, 0, 5], x[4, 0, 6], x[20, 0, 7] = math.inf, -math.inf, math.nan
        x[:16, 0, 8] = 0.0
        nnc.op_kv_write_paged(cache, x, x, _ints(range(40)), _ints([0] * 40))
        bounds = nnc.op_page_bounds(cache, nnc.page_bounds(cache), _ints([40]), _ints([-5]))
        at = cache.page_table[0].long()
        first = bounds[at[0], 0]
        assert first[1, 5] == math.inf and first[0, 6] == -math.inf and (first[:, 8] == 0).all()
        assert bounds[at[1], 0, :, 7].isnan().all() and not bounds[at[1], 0, :, :7].isnan().any() and bounds[at[2]].isfinite().all()
    cache = _paged(nnc, E4M3, [20], 16, 1, 64, 1)
    x = _randn(_gen(1), 20, 1, 64)
    x[2, 0, 9] = math.nan
    nnc.op_kv_write_paged(cache, x, x, _ints(range(20)), _ints([0] * 20))
    bounds = nnc.op_page_bounds(cache, nnc.page_bounds(cache), _ints([20]))
    assert bounds[cache.page_table[0, 0].long(), 0, :, 9].isnan().all() and bounds.isnan().sum() == 2


def test_bounds_of_lengths_and_pages_out_of_range(nnc):
    cache = _paged(nnc, BF16, [48, 48], 16, 2, 64, 6)
    held = _fill(nnc, cache, [48, 48], 1)
    cache.page_table[1, 1] = 99
    cache.page_table[1, 2] = -3
    bounds = nnc.page_bounds(cache).fill_(7.0)
    nnc.op_page_bounds(cache, bounds, _ints([2 ** 31 - 1, 48]))
    assert nnc.op_status() == 0x100
    want = _bounds64(held, [48, 48], 16)
    for i in range(3):
        assert torch.equal(bounds[cache.page_table[0, i].long()].double(), want[0][i])
    assert torch.equal(bounds[cache.page_table[1, 0].long()].double(), want[1][0])
    bounds.fill_(7.0)
    nnc.op_page_bounds(cache, bounds, _ints([-4, 48]), _ints([0, 2 ** 31 - 1]))      # nothing new
    assert (bounds == 7).all() and nnc.op_status() == 0


# ---- scores ----------------------------------------------------------------------------------------------------------

def _check_scores(scores, q, cache, bounds, lens):
    """Against max over the heads of sum max(q lo, q hi).  fp32 part: 2 d / 16 steps of up to three terms each of the tensor cores
    and 8 more of other arithmetic, 2^-22 each of the sum of magnitudes (fp16 terms of fp32 queries leave 2^-22 of their largest
    element, which 8 of these cover: it is at most sqrt(d) times a query's root mean square)."""
    batch, hq, d = q.shape
    for b, n in enumerate(lens):
        pages = -(-n // cache.page_size)
        assert (scores[b, :, pages:] == -math.inf).all()
        if not pages:
            continue
        x = bounds[cache.page_table[b, :pages].long()].double().transpose(0, 1)[:, None]      # [heads][1][pages][2][d]
        y = q[b].double().view(cache.n_kv_heads, -1, 1, d)
        product = torch.maximum(y * x[..., 0, :], y * x[..., 1, :])
        size = product.abs().sum(-1)
        want = product.sum(-1)
        tol = (2.0 ** -22 * (3 * 2 * d / 16 + 8) * size).amax(1)
        bad = (scores[b, :, :pages].double() - want.amax(1)).abs() > tol
        assert not bad.any(), (b, bad.sum().item(), ((scores[b, :, :pages].double() - want.amax(1)).abs() / tol).max().item())


@pytest.mark.parametrize("kv,dtype", TYPES, ids=str)
@pytest.mark.parametrize("heads,group,d,page", [(1, 1, 128, 16), (2, 4, 64, 32), (8, 2, 128, 64), (3, 8, 64, 16), (1, 9, 128, 128), (2, 40, 64, 256)])
def test_scores(nnc, kv, dtype, heads, group, d, page):
    lens = [0, 1, page, page + 1, 16 * page, 17 * page - 1, 5 * page, 90 * page + 3]
    cache = _paged(nnc, kv, [min(n, 2) for n in lens], page, heads, d, 5)         # the scores read no rows
    total = 60
    cache = nnc.PagedKV.empty(total, page, heads, d, kv, len(lens), max(-(-n // page) for n in lens) + 1)
    g = _gen(heads * group)
    cache.page_table[:] = torch.randint(0, total, cache.page_table.shape, generator=g, device="cuda", dtype=torch.int32)
    for b, n in enumerate(lens):
        cache.page_table[b, -(-n // page):] = -1
    bounds = nnc.page_bounds(cache)
    bounds.copy_(_randn(g, total, heads, 1, d) + torch.rand(total, heads, 2, d, generator=g, device="cuda") * torch.tensor([[-1.0], [1.0]], device="cuda"))
    q = _randn(g, len(lens), heads * group, d) * torch.exp2(torch.randint(-9, 9, (len(lens), heads * group, 1), generator=g, device="cuda").float())
    q[2] = 0
    q = q.to(dtype)
    scores = nnc.op_score_pages(q, cache, bounds, _ints(lens))
    assert scores.shape == (len(lens), heads, cache.pages_per_seq) and scores.dtype is F32
    _check_scores(scores, q, cache, bounds, lens)
    assert nnc.op_status() == 0
    wide = torch.cat([q.flatten(1), torch.full((len(lens), 64), math.nan, dtype=dtype, device="cuda")], 1)[:, :heads * group * d].unflatten(1, (heads * group, d))
    assert torch.equal(nnc.op_score_pages(wide, cache, bounds, _ints(lens)), scores)
    assert nnc.op_score_pages(q[:0], cache, bounds, _ints([])).shape == (0, heads, cache.pages_per_seq)


def test_no_key_of_a_page_has_a_larger_product(nnc):
    """The score is a bound: within the arithmetic's error, every product of a query with a key of the page lies below."""
    for kv in (BF16, F16, E4M3):
        lens, page, heads, d = [900, 333], 16, 2, 128
        cache = _paged(nnc, kv, lens, page, heads, d, 1)
        held = _fill(nnc, cache, lens, 2)
        bounds = nnc.op_page_bounds(cache, nnc.page_bounds(cache), _ints(lens))
        q = _randn(_gen(3), 2, heads * 4, d)
        scores = nnc.op_score_pages(q, cache, bounds, _ints(lens))
        _check_scores(scores, q, cache, bounds, lens)
        for b, n in enumerate(lens):
            s = torch.einsum("hgd,hnd->hgn", q[b].double().view(heads, 4, d), held[0][b]).amax(1)
            s = torch.nn.functional.pad(s, (0, -n % page), value=-math.inf).unflatten(1, (-1, page)).amax(-1)
            assert (scores[b, :, :s.shape[1]].double() >= s - 1e-3).all()


def test_scores_of_numbers_that_are_not_finite_and_of_pages_out_of_range(nnc):
    for dtype in (BF16, F32):
        cache = nnc.PagedKV.empty(8, 16, 1, 64, BF16, 1, 8)
        cache.page_table[0] = _ints(range(8))
        bounds = nnc.page_bounds(cache)
        bounds[:, :, 0], bounds[:, :, 1] = -1.0, 2.0
        bounds[1, 0, 1, 3] = math.inf
        bounds[2, 0, :, 4] = math.nan
        bounds[3, 0, 0, 5] = -math.inf
        cache.page_table[0, 6] = 8
        q = _randn(_gen(1), 1, 3, 64).to(dtype)
        scores = nnc.op_score_pages(q, cache, bounds, _ints([8 * 16]))[0, 0]
        assert nnc.op_status() == 0x100
        assert not scores[[1, 2, 3]].isfinite().any() and not (scores[[1, 2, 3]] == -math.inf).any()
        assert scores[6] == -math.inf and scores[[0, 4, 5, 7]].isfinite().all()
        pages, counts = nnc.op_select_pages(scores[None, None].contiguous(), _ints([8 * 16]), 16, 5)
        assert pages.tolist() == [[[0, 1, 2, 3, 7]]] and counts.tolist() == [[5]]
        full = nnc.op_score_pages(q, cache, bounds, _ints([10 ** 9]))
        assert nnc.op_status() == 0x100 and torch.equal(full[0, 0].nan_to_num(nan=5e9), scores.nan_to_num(nan=5e9))


# ---- selection -------------------------------------------------------------------------------------------------------

def _select(scores, lens, page, n, first, last):
    """The definition, row by row."""
    batch, heads, columns = scores.shape
    pages = torch.full((batch, heads, n), -1, dtype=torch.int32)
    counts = torch.zeros(batch, heads, dtype=torch.int32)
    rows = scores.cpu().double()
    for b in range(batch):
        have = min(-(-max(0, lens[b]) // page), columns)
        for h in range(heads):
            x = rows[b, h, :have].clone()
            rank = torch.where(x.isnan(), 1.0, 0.0)                 # 2: always in, 1: NaN, 0: by value
            rank[:first] = 2
            if last and have:
                rank[max(0, have - last):] = 2
            x = torch.where(rank > 0, 0.0, x)
            order = sorted(range(have), key=lambda i: (-rank[i].item(), -x[i].item(), i))
            got = sorted(order[:n])
            pages[b, h, :len(got)] = torch.tensor(got, dtype=torch.int32)
            counts[b, h] = len(got)
    return pages, counts


def _check_selection(nnc, scores, lens, page, n, first=1, last=1):
    pages, counts = nnc.op_select_pages(scores, _ints(lens), page, n, first, last)
    want, want_counts = _select(scores, lens, page, n, first, last)
    assert torch.equal(pages.cpu(), want) and torch.equal(counts.cpu(), want_counts)


@pytest.mark.parametrize("columns,n,first,last", [(1, 1, 0, 0), (1, 1, 1, 0), (1, 8, 1, 1), (2, 1, 0, 1), (40, 7, 1, 1), (40, 40, 2, 5), (300, 299, 0, 0),
                                                  (513, 64, 3, 4), (513, 1, 0, 0), (2049, 256, 1, 1), (4097, 4000, 0, 9), (9000, 2, 1, 1)])
def test_selection(nnc, columns, n, first, last):
    g = _gen(columns + n)
    lens = [0, 1, 32, 33, 32 * columns, 32 * columns - 31, 32 * (columns // 2), 32 * columns + 1000, -7]
    scores = 40 + 12 * _randn(g, len(lens), 3, columns)
    _check_selection(nnc, scores, lens, 32, n, first, last)
    _check_selection(nnc, scores.round(), lens, 32, n, first, last)                          # many equals
    _check_selection(nnc, (scores * 0.02).round() * 0.5 - 0.25, lens, 32, n, first, last)    # both signs, few values
    _check_selection(nnc, torch.zeros_like(scores), lens, 32, n, first, last)
    _check_selection(nnc, torch.where(scores > 40, 0.0, -0.0), lens, 32, n, first, last)     # zeros of either sign are equal
    _check_selection(nnc, scores * 1e-44, lens, 32, n, first, last)                          # subnormals
    odd = scores.clone()
    odd[odd > 55], odd[odd < 20], odd[(odd > 40) & (odd < 41)] = math.inf, -math.inf, math.nan
    _check_selection(nnc, odd, lens, 32, n, first, last)


def test_selection_from_rows_too_long_for_shared_memory(nnc):
    columns = 41003
    scores = _randn(_gen(1), 2, 1, columns)
    scores[1] = scores[1].mul(4).round()
    _check_selection(nnc, scores, [16 * columns, 16 * 41001 - 3], 16, 1000)


def test_selection_of_many_rows(nnc):
    scores = _randn(_gen(2), 700, 2, 70)
    _check_selection(nnc, scores, [(37 * b) % 4600 for b in range(700)], 64, 9, 2, 2)


# ---- attention over listed pages -----------------------------------------------------------------------------------------

def _check_selected(out, lse, q, held, lens, lists, page, scale, kv):
    """lists[b][h]: the pages that count."""
    heads = held[0][0].shape[0]
    group = q.shape[1] // heads
    for b, n in enumerate(lens):
        for h in range(heads):
            at = [i for x in lists[b][h] for i in range(x * page, min(n, (x + 1) * page))]
            part = [[t[b][h:h + 1, at]] for t in held]
            rows = slice(h * group, (h + 1) * group)
            _check_attention(out[b:b + 1, rows], lse[b:b + 1, rows], q[b:b + 1, rows], part, [len(at)], scale, 0, kv)


def _lists(lists, n, fill=-1):
    """(pages, counts) of lists[b][h]; entries behind the count hold `fill`."""
    pages = torch.tensor([[x + [fill] * (n - len(x)) for x in of] for of in lists], dtype=torch.int32, device="cuda")
    return pages, torch.tensor([[len(x) for x in of] for of in lists], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kv,dtype", TYPES, ids=str)
@pytest.mark.parametrize("heads,group,d,page,n", [(1, 1, 128, 16, 5), (2, 4, 128, 64, 3), (8, 2, 64, 32, 9), (1, 8, 64, 256, 2), (2, 7, 128, 128, 4),
                                                  (2, 16, 128, 16, 40), (1, 17, 128, 32, 6), (3, 5, 64, 16, 1), (3, 32, 64, 64, 7)])
def test_attention_over_listed_pages(nnc, scratch, kv, dtype, heads, group, d, page, n):
    lens = [0, 1, 15, 16, 17, 64, 0, 65, 127, 129, 700, 3, 1500]
    cache = _paged(nnc, kv, lens, page, heads, d, heads * 100 + group)
    held = _fill(nnc, cache, lens, group)
    g = torch.Generator().manual_seed(n)
    lists = []
    for b, length in enumerate(lens):
        have = -(-length // page)
        lists.append([])
        for h in range(heads):
            x = torch.randperm(have, generator=g)[:n].tolist()             # in no order
            if (b + h) % 4 == 3:
                x = x[:len(x) // 2]                                        # fewer, or none
            lists[-1].append(x)
    pages, counts = _lists(lists, n, 77)                                   # what lies behind the count may be anything
    q = _randn(_gen(d + group), len(lens), heads * group, d, dtype=dtype)
    out, lse = nnc.op_attn_selected_paged(q, cache, _ints(lens), pages, counts, scratch=scratch, want_lse=True)
    _check_selected(out, lse, q, held, lens, lists, page, d ** -0.5, kv)
    assert nnc.op_status() == 0 and not scratch[:8192].any()
    again = nnc.op_attn_selected_paged(q, cache, _ints(lens), pages, counts, want_lse=True)     # a scratch of the call's own
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (E4M3, F32), (F16, F16)], ids=str)
@pytest.mark.parametrize("batch,heads,group,length,page,n", [(1, 8, 4, 9000, 16, 400), (1, 1, 16, 30011, 256, 100), (200, 2, 2, 333, 32, 8), (37, 4, 3, 1024, 64, 11),
                                                             (20, 1, 16, 2500, 16, 100), (2, 1, 80, 9000, 128, 50)])
def test_listed_pages_split_over_many_and_few_ctas(nnc, scratch, kv, dtype, batch, heads, group, length, page, n):
    lens = [length - (b * 37) % length for b in range(batch)]
    cache = _paged(nnc, kv, lens, page, heads, 128, batch)
    held = _fill(nnc, cache, lens, batch + 1)
    g = torch.Generator().manual_seed(n)
    lists = [[sorted(torch.randperm(-(-x // page), generator=g)[:n].tolist()) for _ in range(heads)] for x in lens]
    q = _randn(_gen(batch), batch, heads * group, 128, dtype=dtype)
    out, lse = nnc.op_attn_selected_paged(q, cache, _ints(lens), *_lists(lists, n), scratch=scratch, want_lse=True, scale=0.2)
    _check_selected(out, lse, q, held, lens, lists, page, 0.2, kv)


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_all_pages_in_order_are_the_whole_sequence(nnc, scratch, kv):
    lens = [1000, 17, 512]
    cache = _paged(nnc, kv, lens, 16, 2, 128, 1)
    _fill(nnc, cache, lens, 2)
    q = _randn(_gen(3), 3, 8, 128, dtype=BF16)
    n = cache.pages_per_seq
    pages = torch.arange(n, device="cuda", dtype=torch.int32).expand(3, 2, n).contiguous()
    got = nnc.op_attn_selected_paged(q, cache, _ints(lens), pages, torch.full((3, 2), n, dtype=torch.int32, device="cuda"), scratch=scratch, want_lse=True)
    want = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    assert nnc.op_status() == 0                                            # entries past a sequence's pages are no error
    # shares of other lengths add in another order: a rounding of the result, and 64 steps of fp32 (2^-18) of its parts
    assert torch.allclose(got[0].float(), want[0].float(), rtol=2.0 ** -7, atol=2.0 ** -14) and torch.allclose(got[1], want[1], rtol=2.0 ** -18, atol=2.0 ** -18)


def test_entries_and_counts_out_of_range(nnc, scratch):
    lens = [100, 100]
    cache = _paged(nnc, BF16, lens, 16, 2, 64, 6)
    held = _fill(nnc, cache, lens, 1)
    q = _randn(_gen(2), 2, 4, 64, dtype=BF16)
    call = lambda pages, counts, at=lens: nnc.op_attn_selected_paged(q, cache, _ints(at), pages, counts, scratch=scratch, want_lse=True)
    lists = [[[0, 3], [6, 1]], [[2], [5, 4]]]
    pages, counts = _lists(lists, 3)
    for bad in (-1, -2 ** 31, 7, 2 ** 31 - 1):                             # no such entry of the table
        wrong = pages.clone()
        wrong[0, 0, 2], wrong[1, 1, 2] = bad, bad
        out, lse = call(wrong, torch.tensor([[3, 2], [1, 3]], dtype=torch.int32, device="cuda"))
        assert nnc.op_status() == 0x100
        _check_selected(out, lse, q, held, lens, lists, 16, 0.125, BF16)
    all_three = [[[0, 3, 2], [6, 1, 0]], [[2, 3, 4], [5, 4, 0]]]
    pages, counts = _lists(all_three, 3)
    out, lse = call(pages, counts + 2 ** 30)                               # counts past the list
    assert nnc.op_status() == 0
    _check_selected(out, lse, q, held, lens, all_three, 16, 0.125, BF16)
    out, lse = call(pages, counts, [100, 33])                              # pages past the length hold nothing
    assert nnc.op_status() == 0
    _check_selected(out, lse, q, held, [100, 33], all_three, 16, 0.125, BF16)
    out, lse = call(pages, counts - 5, [100, 0])
    assert (out == 0).all() and (lse == -math.inf).all() and nnc.op_status() == 0
    out, lse = call(pages, counts, [2 ** 31 - 1, 100])                     # the longest that the table holds: rows of NaN behind 100
    assert nnc.op_status() == 0x100
    cache.page_table[0, 3] = 1 << 30                                       # a page that the pool does not have
    out, lse = call(pages, counts)
    assert nnc.op_status() == 0x100
    _check_selected(out, lse, q, held, lens, [[[0, 2], [6, 1, 0]], all_three[1]], 16, 0.125, BF16)
    assert nnc.op_status() == 0 and not scratch[:8192].any()


@pytest.mark.parametrize("kv", [BF16, F16], ids=str)
def test_infinite_values_in_listed_and_in_other_pages(nnc, scratch, kv):
    lens = [200]
    cache = _paged(nnc, kv, lens, 16, 1, 64, 1)
    g = _gen(1)
    k, v = (_randn(g, 200, 1, 64) for _ in range(2))
    v[17, 0, 3], v[100, 0, 4], v[40, 0, 5], v[199, 0, 6], v[50, 0, 7], v[120, 0, 7] = math.inf, math.inf, -math.inf, math.nan, math.inf, -math.inf
    k[70], v[70] = math.nan, math.nan                                      # in a page that is not listed
    nnc.op_kv_write_paged(cache, k, v, _ints(range(200)), _ints([0] * 200))
    pages, counts = _lists([[[12, 1, 2, 3, 7]]], 6)                        # rows 192-199 and 16-63 and 112-127
    out = nnc.op_attn_selected_paged(_randn(g, 1, 2, 64).to(kv), cache, _ints(lens), pages, counts, scratch=scratch)[0]
    assert (out[:, 3] == math.inf).all() and (out[:, 5] == -math.inf).all() and out[:, 6:8].isnan().all()
    assert out[:, [i for i in range(64) if i not in (3, 5, 6, 7)]].isfinite().all()


# ---- together ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_a_captured_step_that_chooses_its_pages(nnc, scratch, kv):
    """Append, bounds, scores, selection, attention: captured once, replayed while positions and lengths move on; beside it the same
    on a stream of its own with a scratch of its own.  Every replay's selection is the one that its scores define, its scores those of
    its bounds, and its attention that over its selection."""
    heads, group, d, page, n, steps = 2, 4, 64, 16, 6, 20
    start = [0, 13, 130, 400]
    batch, most = len(start), 500
    g = _gen(5)
    stream_k, stream_v, stream_q = (_randn(g, batch, most, x, d, dtype=BF16) for x in (heads, heads, heads * group))
    held = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    sides = []
    for side in range(2):
        cache = _paged(nnc, kv, [x + steps for x in start], page, heads, d, side)
        bounds = nnc.page_bounds(cache)
        for b, x in enumerate(start):
            p = torch.arange(x, device="cuda", dtype=torch.int32)
            nnc.op_kv_write_paged(cache, stream_k[b, :x].contiguous(), stream_v[b, :x].contiguous(), p, torch.full_like(p, b))
        nnc.op_page_bounds(cache, bounds, _ints(start))
        pos, lens = _ints(start), _ints(start)
        buffers = [torch.empty(batch, x, d, dtype=BF16, device="cuda") for x in (heads, heads, heads * group)]
        own = scratch if side == 0 else nnc.attn_paged_scratch()

        def step(cache=cache, bounds=bounds, pos=pos, lens=lens, buffers=buffers, own=own):
            nnc.op_kv_write_paged(cache, buffers[0], buffers[1], pos)
            lens.copy_(pos + 1)
            nnc.op_page_bounds(cache, bounds, lens, pos)
            scores = nnc.op_score_pages(buffers[2], cache, bounds, lens)
            pages, counts = nnc.op_select_pages(scores, lens, page, n)
            out, lse = nnc.op_attn_selected_paged(buffers[2], cache, lens, pages, counts, scratch=own, want_lse=True)
            pos.add_(1)
            return scores, pages, counts, out, lse

        for t, source in zip(buffers, (stream_k, stream_v, stream_q)):
            t.copy_(source[torch.arange(batch), start])
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()                       # once without a capture; the same rows are written again below
            pos.copy_(_ints(start))
            graph = torch.cuda.CUDAGraph()
            stream.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                results = step()
        sides.append((graph, stream, cache, bounds, buffers, results, step))     # (step keeps what the graph reads)
    for i in range(steps):
        for graph, stream, cache, bounds, buffers, *_ in sides:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for t, source in zip(buffers, (stream_k, stream_v, stream_q)):
                    t.copy_(source[torch.arange(batch), [x + i for x in start]])
                graph.replay()
        torch.cuda.synchronize()
        lens = [x + i + 1 for x in start]
        rows = [[held(t[b, :x]).transpose(0, 1) for b, x in enumerate(lens)] for t in (stream_k, stream_v)]
        for _, _, cache, bounds, buffers, (scores, pages, counts, out, lse), _ in sides:
            for b, of in enumerate(_bounds64(rows, lens, page)):
                for j, x in enumerate(of):
                    assert torch.equal(bounds[cache.page_table[b, j].long()].double(), x)
            _check_scores(scores, buffers[2], cache, bounds, lens)
            want, want_counts = _select(scores, lens, page, n, 1, 1)
            assert torch.equal(pages.cpu(), want) and torch.equal(counts.cpu(), want_counts)
            lists = [[want[b, h, :want_counts[b, h]].tolist() for h in range(heads)] for b in range(batch)]
            _check_selected(out, lse, buffers[2], rows, lens, lists, page, d ** -0.5, kv)
    assert nnc.op_status() == 0


def test_refusals_of_the_binding(nnc, scratch):
    cache = _paged(nnc, BF16, [40, 40], 16, 2, 64, 1)
    _fill(nnc, cache, [40, 40], 2)
    q, lens = _randn(_gen(1), 2, 4, 64, dtype=BF16), _ints([40, 40])
    bounds = nnc.page_bounds(cache)
    pages, counts = _lists([[[0], [1]], [[0], [1]]], 2)
    call = nnc.op_attn_selected_paged
    other = nnc.page_bounds(_paged(nnc, F16, [40, 40], 16, 2, 64, 1))
    for refused in (lambda: nnc.op_page_bounds(cache, other, lens), lambda: nnc.op_page_bounds(cache, bounds[:-1], lens),
                    lambda: nnc.op_page_bounds(cache, bounds.cpu(), lens), lambda: nnc.op_page_bounds(cache, bounds, lens.long()),
                    lambda: nnc.op_page_bounds(cache, bounds, lens, lens[:1]), lambda: nnc.op_page_bounds(cache, bounds.transpose(1, 2), lens),
                    lambda: nnc.op_page_bounds(cache, cache.k.view(-1)[:bounds.numel()].view_as(bounds), lens),
                    lambda: nnc.op_page_bounds(cache, bounds.clone().requires_grad_(), lens),
                    lambda: nnc.op_score_pages(q[..., :32], cache, bounds, lens), lambda: nnc.op_score_pages(q, cache, bounds, lens[:1]),
                    lambda: nnc.op_score_pages(q, cache, bounds.float(), lens), lambda: nnc.op_score_pages(q.cpu(), cache, bounds, lens),
                    lambda: nnc.op_select_pages(torch.zeros(2, 2, 3), lens, 16, 2), lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda"), lens, 16, 0),
                    lambda: nnc.op_select_pages(torch.zeros(2, 3, device="cuda"), lens, 16, 2), lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda").half(), lens, 16, 2),
                    lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda"), lens, 16, 2, -1), lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda"), lens, 16, 1 << 40),
                    lambda: call(q, cache, lens, pages.long(), counts), lambda: call(q, cache, lens, pages[:1], counts), lambda: call(q, cache, lens, pages, counts[:, :1]),
                    lambda: call(q, cache, lens, pages[..., :0], counts), lambda: call(q, cache, lens, pages[..., :1], counts), lambda: call(q, cache, lens, pages.cpu(), counts),
                    lambda: call(q, cache, lens, pages, counts, out=q[:, :2]), lambda: call(q, cache, lens, pages, counts, scratch=scratch.cpu()),
                    lambda: call(q, cache, lens, pages, counts, out=cache.k.view(-1)[:q.numel()].view_as(q))):
        with pytest.raises(ValueError):
            refused()
    with pytest.raises(TypeError):
        nnc.op_page_bounds(cache, None, lens)
    for refused, status in ((lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda"), lens, 16, 2, 2, 1), -1),
                            (lambda: nnc.op_select_pages(torch.zeros(2, 2, 3, device="cuda"), lens, 48, 2), -1),
                            (lambda: nnc.op_score_pages(q.half(), cache, bounds, lens), -1), (lambda: call(q, cache, lens, pages, counts, scratch=scratch[:1 << 20]), -2),
                            (lambda: nnc.op_score_pages(_randn(_gen(1), 2, 258, 64, dtype=BF16), cache, bounds, lens), -3)):
        with pytest.raises(nnc.NncError) as e:
            refused()
        assert e.value.status == status
    before = bounds._version
    nnc.op_page_bounds(cache, bounds, lens)
    assert bounds._version == before + 1
    same = q.clone()
    assert call(same, cache, lens, pages, counts, out=same, scratch=scratch) is same
    assert torch.equal(same, call(q, cache, lens, pages, counts, scratch=scratch))


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_pages_far_in_a_pool_of_more_than_32_bits_of_elements(nnc, scratch, kv):
    """The same rows at the pool's beginning and past its 2^31st (of codes: 2^32nd) element: the same results bit for bit."""
    page, heads, d, lens, common = 256, 4, 128, [1100, 1024, 1290, 1030], 1024
    whole, own = common // page, [-(-(n - common) // page) for n in lens]
    far = (1 << (32 if kv is E4M3 else 31)) // (page * heads * d) + 3
    results = []
    for first in (1, far):
        cache = nnc.PagedKV.empty(first + whole + sum(own), page, heads, d, kv, len(lens), 200)
        at = first + whole
        for b, x in enumerate(own):
            cache.page_table[b, :whole] = torch.arange(first, first + whole, device="cuda")
            cache.page_table[b, whole:whole + x] = torch.arange(at, at + x, device="cuda")
            at += x
        tokens = [(i, 0) for i in range(common)] + [(i, b) for b, n in enumerate(lens) for i in range(common, n)]
        k, v = (_randn(_gen(s), len(tokens), heads, d, dtype=BF16) for s in (1, 2))
        nnc.op_kv_write_paged(cache, k, v, _ints([t[0] for t in tokens]), _ints([t[1] for t in tokens]))
        q, ends = _randn(_gen(3), len(lens), heads * 4, d, dtype=BF16), _ints(lens)
        bounds = nnc.op_page_bounds(cache, nnc.page_bounds(cache), ends)
        scores = nnc.op_score_pages(q, cache, bounds, ends)
        pages, counts = nnc.op_select_pages(scores, ends, page, 3)
        results.append([scores, pages, counts, *nnc.op_attn_selected_paged(q, cache, ends, pages, counts, scratch=scratch, want_lse=True),
                        *nnc.op_attn_prefix_paged(q, cache, ends, _ints([0, 4]), _ints([common]), want_lse=True)])
        assert nnc.op_status() == 0
        del cache, bounds
    for a, b in zip(*results):
        assert torch.equal(a, b) and not a.float().isnan().any()
