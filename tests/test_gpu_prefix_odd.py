"""Numbers that are not finite behind shared prefixes: what the ordinary attention over the same rows makes of them, and at what cost."""
import math

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, _gen, _ints, _randn, nnc  # noqa: F401
from test_gpu_prefix import _grouped

pytestmark = pytest.mark.gpu


def _document(nnc, n, members, heads, d, kv, tail):
    """One group behind n positions, normal values everywhere."""
    page = 128
    whole, own = n // page, -(-tail // page)
    cache = nnc.PagedKV.empty(whole + members * own, page, heads, d, kv, members, whole + own)
    for pool, seed in ((cache.k, 1), (cache.v, 2)):
        pool.copy_(_randn(_gen(seed), *pool.shape, dtype=kv))
    cache.page_table[:, :whole] = torch.arange(whole, device="cuda")
    cache.page_table[:, whole:] = whole + torch.arange(members * own, device="cuda").view(members, own)
    return cache, _ints([n + tail] * members), _ints([0, members]), _ints([n])


def _microseconds(call):
    for _ in range(2):
        call()
    times = []
    for _ in range(5):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        call()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end) * 1e3)
    return sorted(times)[2]


@pytest.mark.parametrize("kv,d", [(BF16, 128), (F16, 64)], ids=str)
def test_a_query_without_a_number_and_an_infinite_value_cost_little(nnc, kv, d):
    """65536 shared positions.  A query of NaN is NaN whatever the values are: nothing is looked through for it.  An infinite value makes every share
    look through its own rows once more, which is less than reading all of them was.  (20 us: the host's part of a call.)"""
    cache, lens, starts, shared = _document(nnc, 65536, 16, 2, d, kv, 100)
    q = _randn(_gen(3), 16, 24, d, dtype=kv)
    scratch = nnc.attn_prefix_scratch(16, 24, d)
    call = lambda q: nnc.op_attn_prefix_paged(q, cache, lens, starts, shared, scratch=scratch)
    plain, out = _microseconds(lambda: call(q)), call(q)
    nan_q = q.clone()
    nan_q[5, 3] = math.nan
    assert _microseconds(lambda: call(nan_q)) < 1.5 * plain + 20
    got = call(nan_q)
    assert got[5, 3].isnan().all()
    got[5, 3] = out[5, 3]
    assert torch.equal(got, out)
    cache.v[200, 1, 5, 7] = math.inf
    assert _microseconds(lambda: call(q)) < 4 * plain + 20
    got = call(q)
    assert (got[:, 12:, 7] == math.inf).all()
    got[:, 12:, 7] = out[:, 12:, 7]
    assert torch.equal(got, out)


@pytest.mark.parametrize("kv,d", [(BF16, 128), (F16, 64), (BF16, 64)], ids=str)
def test_columns_are_the_ordinary_attention_s(nnc, kv, d):
    """Infinities of either sign and NaN among values, keys that put whole shares out of sight, on both sides of the prefix's end: the same columns
    come out infinite, of the same sign, or as no number."""
    groups = [(4096, [4100, 4200, 4096, 900]), (640, [700, 701])]
    for seed in range(6):
        cache, lens, starts, shared, _ = _grouped(nnc, kv, groups, 32, 2, d, seed)
        r = torch.Generator().manual_seed(seed)
        draw = lambda n: int(torch.randint(0, n, (1,), generator=r))
        at = lambda b, pos: (cache.page_table[b, pos // 32].long(), draw(2), pos % 32)
        for i in range(3 * seed):
            b = draw(len(lens))
            cache.v[(*at(b, draw(lens[b])), draw(d))] = (math.inf, -math.inf, math.nan)[draw(3)]
        lo = 64 * draw(20)
        for pos in range(lo, lo + 64 * (5 + 8 * seed)):                    # seed 5: 45 steps
            page, _, slot = at(0, pos)
            cache.k[page, :, slot, 0] = -math.inf
        page, head, slot = at(0, lo + 70)
        cache.v[page, head, slot, 1] = math.inf                            # a row whose weight is 0, in a share where all are
        q = _randn(_gen(seed), len(lens), 10, d, dtype=kv)
        q[..., 0] = q[..., 0].abs() + 0.1
        out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
        want, want_lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), want_lse=True)
        kind = lambda x: torch.where(x.isnan(), 3, torch.where(x == math.inf, 1, torch.where(x == -math.inf, 2, 0)))
        assert torch.equal(kind(out), kind(want)) and (kind(out) == 1).any(), seed
        here = out.isfinite()
        # a rounding each of the result, and fp32 sums and two terms of the weights
        assert torch.allclose(out[here].float(), want[here].float(), rtol=torch.finfo(kv).eps, atol=2.0 ** -10)
        assert torch.allclose(lse, want_lse, rtol=2.0 ** -18, atol=2.0 ** -18)
    assert nnc.op_status() == 0


@pytest.mark.parametrize("kv,d", [(BF16, 128), (F16, 64), (E4M3, 128), (E4M3, 64)], ids=str)
def test_weights_between_prefix_and_tail_are_exact_where_scores_are(nnc, kv, d):
    """Every score is 2^14 (times a scale of 1: an exact product in log2 units, too), values are 1 in the prefix and -1 behind it: every weight is 1, and a
    result differs from the counts' quotient by its own rounding, and 2^-16 for two terms of the weights, however large the scores are."""
    shared, tails = 640, [640, 64, 1, 639, 5000]
    cache, lens, starts, groups, _ = _grouped(nnc, kv, [(shared, [shared + t for t in tails])], 32, 1, d, 1)
    k = torch.zeros(max(lens), 1, d, device="cuda")
    k[:, 0, 0] = 1.0
    v = torch.ones_like(k)
    v[shared:] = -1.0
    for b, n in enumerate(lens):
        first = 0 if b == 0 else shared
        nnc.op_kv_write_paged(cache, k[first:n].contiguous(), v[first:n].contiguous(), _ints(range(first, n)), _ints([b] * (n - first)))
    q = torch.zeros(len(lens), 3, d, dtype=F16 if kv is F16 else BF16, device="cuda")
    q[..., 0] = 2.0 ** 14
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(groups), scale=1.0, want_lse=True)
    for b, t in enumerate(tails):
        want = (shared - t) / (shared + t)
        assert ((out[b].double() - want).abs() <= torch.finfo(out.dtype).eps / 2 * abs(want) + 2.0 ** -16).all(), (b, out[b, 0, 0].item(), want)
        # the weights' reference and the result's own rounding: two half steps of 2^-9 (values up to 2^15)
        assert ((lse[b].double() - (2.0 ** 14 + math.log(shared + t))).abs() <= 2.0 ** -9 + 2.0 ** -16).all()


@pytest.mark.parametrize("kv,d", [(BF16, 128), (F16, 64)], ids=str)
def test_an_infinity_behind_the_prefix_whose_row_weighs_nothing(nnc, kv, d):
    """All keys behind the prefix are out of sight (scores of -infinity) and one of their values is infinite: its column is, as in the ordinary attention."""
    cache, lens, starts, shared, _ = _grouped(nnc, kv, [(640, [700, 650, 640])], 32, 1, d, 4)
    for pos in range(640, 700):
        cache.k[cache.page_table[0, pos // 32].long(), :, pos % 32, 0] = -math.inf
    cache.v[cache.page_table[0, 20].long(), 0, 9, 3] = -math.inf
    q = _randn(_gen(5), 3, 4, d).abs().to(kv)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
    want, want_lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), want_lse=True)
    assert (want[0, :, 3] == -math.inf).all() and torch.equal(out.isfinite(), want.isfinite()) and (out[0, :, 3] == -math.inf).all()
    assert torch.allclose(lse, want_lse, rtol=2.0 ** -18, atol=2.0 ** -18)
