"""Which groups' rows are read for all of their sequences at once: it is the first sequence's pages that are read then, which shows here as the other
sequences' own pages, of other values, not counting."""
import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, _check_attention, _gen, _ints, _randn, nnc, quantise64  # noqa: F401
from test_gpu_prefix import _grouped

pytestmark = pytest.mark.gpu


def _two_sides(nnc, kv, members, group, d, n_groups, seed=1):
    """One group of `members` behind 512 positions, and one sequence of no group; every member but the first has shared pages of its own with other
    values.  The results, and those over the first sequence's pages and over each one's own."""
    page, heads, shared = 64, 2, 512
    cache, lens, starts, _, held = _grouped(nnc, kv, [(shared, [shared + 9 + 20 * i for i in range(members)]), (0, [300])], page, heads, d, seed, spare=8 * members)
    batch = members + 1
    own = [[x.clone() for x in side] for side in held]
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    used = set(cache.page_table[cache.page_table >= 0].tolist()) if cache.page_table.min() < 0 else {p for b, n in enumerate(lens) for p in cache.page_table[b, :-(-n // page)].tolist()}
    free = [p for p in range(cache.n_pages) if p not in used]
    g = _gen(seed + 9)
    for b in range(1, members):
        cache.page_table[b, :8] = _ints([free.pop() for _ in range(8)])
        k, v = (_randn(g, shared, heads, d) for _ in range(2))
        nnc.op_kv_write_paged(cache, k, v, _ints(range(shared)), _ints([b] * shared))
        for which, x in enumerate((k, v)):
            own[which][b][:, :shared] = hold(x).transpose(0, 1)
    q = _randn(_gen(seed + 1), batch, heads * group, d, dtype=F16 if kv is F16 else BF16)
    at = [0, members] + [members] * (n_groups - 1)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(at), _ints([shared] * n_groups), want_lse=True)
    assert nnc.op_status() == 0
    check = lambda side: _check_attention(out, lse, q, side, lens, d ** -0.5, 0, kv)
    return check, held, own


@pytest.mark.parametrize("kv", [BF16, F16, E4M3], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_groups_without_sequences_do_not_turn_sharing_off(nnc, kv, d):
    """As many groups as sequences, all but the first empty: what a captured step has that keeps room for any number of groups."""
    for n_groups in (1, 3, 6):
        check, first_s, _ = _two_sides(nnc, kv, 5, 4, d, n_groups)
        check(first_s)


@pytest.mark.parametrize("kv,members,group,at_once", [(BF16, 2, 1, True), (F16, 2, 4, True), (E4M3, 2, 4, False), (E4M3, 3, 15, False), (E4M3, 3, 16, True), (E4M3, 4, 1, True),
                                                      (E4M3, 2, 23, False), (E4M3, 2, 24, True)], ids=str)
def test_groups_of_few_sequences(nnc, kv, members, group, at_once):
    check, first_s, own = _two_sides(nnc, kv, members, group, 64, 1)
    check(first_s if at_once else own)


@pytest.mark.parametrize("kv,group", [(BF16, 4), (BF16, 31), (BF16, 32), (E4M3, 47), (E4M3, 48)], ids=str)
def test_groups_of_one(nnc, kv, group):
    """As many as sequences, on both sides of where their rows go through the prefix's kernel."""
    cache, lens, starts, shared, held = _grouped(nnc, kv, [(512, [513 + 30 * i]) for i in range(5)], 64, 2, 128, 3)
    q = _randn(_gen(4), 5, 2 * group, 128, dtype=BF16)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
    _check_attention(out, lse, q, held, lens, 128 ** -0.5, 0, kv)
    assert nnc.op_status() == 0


def test_a_refused_call_launches_nothing(nnc):
    """A table of more positions than the rows behind prefixes are counted in: refused as the ordinary attention refuses it, before the first launch."""
    batch, heads = 128, 64
    cache = nnc.PagedKV.empty(1, 256, heads, 64, BF16, batch, 65600)
    q = _randn(_gen(1), batch, heads, 64, dtype=BF16)
    scratch = torch.zeros_like(nnc.attn_prefix_scratch(batch, heads, 64))
    for call in (lambda: nnc.op_attn_prefix_paged(q, cache, _ints([0] * batch), _ints([0, batch]), _ints([0]), scratch=scratch),
                 lambda: nnc.op_attn_decode_paged(q, cache, _ints([0] * batch), scratch=scratch)):
        with pytest.raises(nnc.NncError) as e:
            call()
        assert e.value.status == -3 and not scratch.any()


def test_queries_without_heads_are_refused_as_the_ordinary_attention_refuses_them(nnc):
    cache, lens, starts, shared, _ = _grouped(nnc, BF16, [(32, [40, 40])], 16, 2, 64, 1)
    q = _randn(_gen(1), 2, 0, 64, dtype=BF16)
    for call in (lambda: nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared)), lambda: nnc.op_attn_decode_paged(q, cache, _ints(lens))):
        with pytest.raises(nnc.NncError) as e:
            call()
        assert e.value.status == -1
