"""Attention behind shared prefixes on E4M3 caches, whose kernel converts codes, holds half of a step's scores at a time and has its own
columns for the terms of the weights: the scores, pages, shares and groups that the 16-bit forms are tested with, against 64 bits.

The weights are two bf16 terms here, each off by half a step of what the one before it leaves: 2^-8 * 2^-8 = 2^-16 of a weight.  The rest of
the bounds is _check_attention's."""
import math

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, _gen, _ints, _randn, attend64, nnc, quantise64  # noqa: F401
from test_gpu_prefix import _grouped

pytestmark = pytest.mark.gpu


def _check_codes(out, lse, q, held, lens, scale):
    k, v = held
    d, u = q.shape[-1], 2.0 ** -22
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        want, want_lse, size, reach = attend64(q[b], k[b], v[b], scale, 0)
        score, sums = u * (3 * d / 16 + 8) * reach, u * (n / 16 + 32)
        tol = torch.finfo(out.dtype).eps / 2 * want.abs() + (2.0 ** -16 + sums + 2 * score)[..., None] * size
        bad = (out[b].double() - want).abs() > tol
        assert not bad.any(), (b, n, bad.sum().item(), ((out[b].double() - want).abs() / tol).max().item())
        bad = (lse[b].double() - want_lse).abs() > score + sums + 2.0 ** -22 * want_lse.abs()
        assert not bad.any(), (b, n, (lse[b].double() - want_lse).abs().max().item())


def _case(nnc, groups, page, heads, group, d, seed=1, scale=None, change=None):
    cache, lens, starts, shared, held = _grouped(nnc, E4M3, groups, page, heads, d, seed)
    q = _randn(_gen(seed + 1), len(lens), heads * group, d)
    q = (q if change is None else change(q)).to(BF16)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), scale=scale, want_lse=True)
    _check_codes(out, lse, q, held, lens, d ** -0.5 if scale is None else scale)
    assert nnc.op_status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_peaked_flat_and_extreme_scores_of_codes(nnc, d):
    def change(q):
        q[0] = 0                       # all scores alike
        q[1] *= 30                     # a few positions carry everything
        q[2] *= 1e-6
        q[3, :, 0] = 300.0             # one element above the others
        return q
    for scale in (None, 0.0, -0.3, 1e-30, 4.0):
        _case(nnc, [(640, [700, 650, 641, 640, 900, 333])], 32, 2, 4, d, scale=scale, change=change)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("falls", [False, True])
def test_scores_of_codes_that_grow_or_fall_with_the_position(nnc, d, falls):
    """The reference moves at every step, or never after the first; steps of one team that the other's reference is far from."""
    n, members = 2560, 5
    cache, lens, starts, shared, _ = _grouped(nnc, E4M3, [(n, [n + 1 + 40 * i for i in range(members)])], 32, 1, d, 3)
    most = max(lens)
    k, v = (_randn(_gen(4), most, 1, d) for _ in range(2))
    at = torch.arange(most, device="cuda")
    k[:, 0, 0] = 0.25 * (most - at if falls else at)
    held = [[], []]
    for b, length in enumerate(lens):
        first = 0 if b == 0 else n
        nnc.op_kv_write_paged(cache, k[first:length].contiguous(), v[first:length].contiguous(), _ints(range(first, length)), _ints([b] * (length - first)))
        for which, x in enumerate((k, v)):
            held[which].append(quantise64(x[:length])[0].transpose(0, 1))
    q = _randn(_gen(5), members, 3, d)
    q[..., 0] = 2.0
    q[1, :, 0] = -2.0
    q[2, :, 0] = 0.125
    q = q.to(BF16)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True, scale=1.0)
    _check_codes(out, lse, q, held, lens, 1.0)


@pytest.mark.parametrize("kv", [BF16, F16, E4M3], ids=str)
@pytest.mark.parametrize("page,missing", [(16, [0, 5, 6, 7, 39]), (32, [3, 8, 19]), (64, [0, 4]), (256, [1])])
def test_results_without_the_shared_pages_that_the_pool_does_not_have(nnc, kv, page, missing):
    shared, dtype = 1280 // page * page, F16 if kv is F16 else BF16
    cache, lens, starts, groups, held = _grouped(nnc, kv, [(shared, [shared + 3, shared + 70, shared]), (page, [page + 1])], page, 2, 128, 6)
    for i, at in enumerate(missing):
        cache.page_table[:3, at] = (-1, 1 << 30, cache.n_pages, -2 ** 31)[i % 4]
    gone = {p for at in missing for p in range(at * page, (at + 1) * page)}
    for which in range(2):
        for b in range(3):
            held[which][b] = held[which][b][:, [p for p in range(lens[b]) if p not in gone]]
    q = _randn(_gen(7), 4, 10, 128, dtype=dtype)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(groups), want_lse=True)
    assert nnc.op_status() == 0x100
    _check_codes(out, lse, q, held, [n - len(gone) if b < 3 else n for b, n in enumerate(lens)], 128 ** -0.5)


@pytest.mark.parametrize("heads,group,d,page,shared,members", [(2, 12, 64, 128, 65536, 24), (1, 128, 64, 64, 20000, 7), (4, 30, 128, 32, 9000, 25), (8, 1, 64, 16, 8192, 65)])
def test_long_shares_of_several_tiles_of_codes(nnc, heads, group, d, page, shared, members):
    _case(nnc, [(shared, [shared // page * page + 1 + 3 * i for i in range(members)])], page, heads, group, d)


@pytest.mark.parametrize("d", [64, 128])
def test_many_groups_of_codes(nnc, d):
    _case(nnc, [(16 * (g % 9), [16 * (g % 9) + 1 + (i + g) % 30 for i in range(g % 4)]) for g in range(3, 150)], 16, 2, 4, d)


@pytest.mark.parametrize("d", [64, 128])
def test_shared_codes_behind_a_sequence_s_end_do_not_reach_it(nnc, d):
    for shared, lens_of in ((128, [140, 40, 127, 0, 128]), (4096, [4100, 4095, 70])):
        cache, lens, starts, groups, held = _grouped(nnc, E4M3, [(shared, lens_of)], 16, 2, d, 2)
        last = cache.page_table[0, shared // 16 - 1].long()
        cache.v.view(torch.uint8)[last, :, 15, 4] = 0x7f                   # NaN
        cache.k.view(torch.uint8)[last, :, 15, 0] = 0x7f
        q = _randn(_gen(4), len(lens), 6, d, dtype=BF16)
        out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(groups), want_lse=True)
        short = [b for b, n in enumerate(lens) if n < shared]
        _check_codes(out[short], lse[short], q[short], [[t[b] for b in short] for t in held], [lens[b] for b in short], d ** -0.5)
        assert out[[b for b in range(len(lens)) if b not in short]].isnan().all()


@pytest.mark.parametrize("d", [64, 128])
def test_results_of_long_prefixes_of_codes_are_rounded_once(nnc, d):
    """As of 16-bit caches: the error's root mean square is within a tenth of the rounding's own."""
    n, members = 65536, 4
    cache, lens, starts, shared, held = _grouped(nnc, E4M3, [(n, [n + 1] * members)], 256, 1, d, 5)
    q = _randn(_gen(6), members, 128 // members * 12, d, dtype=BF16)
    out = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared))
    for b in range(members):
        want = torch.softmax(torch.einsum("gd,nd->gn", q[b].double(), held[0][b][0]) * d ** -0.5, -1) @ held[1][b][0]
        error, rounding = (out[b].double() - want).norm(), (want.to(BF16).double() - want).norm()
        assert error < 1.1 * rounding, (b, (error / rounding).item())
