"""Attention of a batch whose sequences share prefixes, against the plain 64-bit form of every sequence's own attention.  Bounds of errors
as in test_gpu_paged, whose own are for one term less of the weights than the kernel has."""
import math

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, F32, TYPES, _check_attention, _gen, _ints, _randn, nnc, quantise64  # noqa: F401

pytestmark = pytest.mark.gpu


def _grouped(nnc, kv, groups, page, heads, d, seed, spare=2, wide=True):
    """groups: (shared positions, lengths of its sequences).  The cache (unused rows NaN), lengths, starts, shared, and what every
    sequence's rows are, 64 bits: two lists of [heads][n][d].  All shared rows are written, whatever the lengths."""
    lens = [n for _, of in groups for n in of]
    starts = [0]
    for _, of in groups:
        starts.append(starts[-1] + len(of))
    whole = [p // page for p, _ in groups]                        # shared pages
    own = [max(0, -(-n // page) - whole[g]) for g, (_, of) in enumerate(groups) for n in of]
    total = sum(whole) + sum(own) + spare
    columns = max(max(-(-max(n, p) // page) for n in of) if of else 0 for p, of in groups) + 1
    if wide:   # a table that could hold enough for the shared rows to be read once; otherwise small batches read them for each sequence
        columns = max(columns, 150_000_000 // (2 * max(1, len(lens)) * page * heads * d))
    cache = nnc.PagedKV.empty(total, page, heads, d, kv, max(1, len(lens)), max(1, columns))
    for pool in (cache.k, cache.v):
        pool.view(torch.uint8).fill_(0x7f) if kv is E4M3 else pool.fill_(math.nan)
    g = _gen(seed)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).int()
    at = 0
    held = [[], []]
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    for i, (p, of) in enumerate(groups):
        common = order[at:at + whole[i]]
        at += whole[i]
        n0 = whole[i] * page
        rows = [_randn(g, n0, heads, d) for _ in range(2)]
        for b in range(starts[i], starts[i + 1]):
            cache.page_table[b, :whole[i]] = common
            cache.page_table[b, whole[i]:whole[i] + own[b]] = order[at:at + own[b]]
            at += own[b]
            n = max(lens[b], n0 if b == starts[i] else 0)
            tail = [_randn(g, max(0, n - n0), heads, d) for _ in range(2)]
            first = 0 if b == starts[i] else n0
            if n > first:
                nnc.op_kv_write_paged(cache, *(torch.cat([x, y])[first:].contiguous() for x, y in zip(rows, tail)), _ints(range(first, n)), _ints([b] * (n - first)))
            for which in range(2):
                held[which].append(hold(torch.cat([rows[which], tail[which]])[:lens[b]]).transpose(0, 1))
    return cache, lens, starts, [p for p, _ in groups], held


def _check(nnc, kv, dtype, groups, page, heads, group, d, seed=1, scale=None, change=None, wide=True):
    cache, lens, starts, shared, held = _grouped(nnc, kv, groups, page, heads, d, seed, wide=wide)
    q = _randn(_gen(seed + 1), len(lens), heads * group, d)
    if change is not None:
        q = change(q)
    q = q.to(dtype)
    scratch = nnc.attn_prefix_scratch(len(lens), heads * group, d)
    call = lambda **kw: nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), scale=scale, want_lse=True, **kw)
    out, lse = call(scratch=scratch)
    _check_attention(out, lse, q, held, lens, d ** -0.5 if scale is None else scale, 0, kv)
    assert nnc.op_status() == 0 and not scratch[:8192].any()
    again = call()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    return out


@pytest.mark.parametrize("kv,dtype", TYPES, ids=str)
@pytest.mark.parametrize("heads,group,d,page", [(1, 1, 128, 16), (2, 4, 128, 64), (8, 2, 64, 32), (1, 8, 64, 256), (2, 7, 128, 128), (3, 17, 64, 16)])
def test_groups_of_any_size(nnc, kv, dtype, heads, group, d, page):
    groups = [(3 * page, [3 * page + 1, 4 * page, 3 * page + 130, 3 * page, 5, 0, 2 * page + 3]),     # lengths below the prefix, none at all
              (page, [page + 7]),                                                                  # one sequence
              (0, [1, 70, 0]),                                                                     # nothing shared
              (2 * page + page // 2, [3 * page, 2 * page + 5]),                                    # not whole pages
              (page - 1, [page, 4]),                                                               # less than one
              (5 * page, [5 * page + i for i in range(40)]),
              (page, [0, 0])]
    for wide in (True, False):
        _check(nnc, kv, dtype, groups, page, heads, group, d, wide=wide)


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)], ids=str)
@pytest.mark.parametrize("heads,group,d,page,shared,members,tail", [(8, 4, 128, 64, 4096, 33, 90), (1, 1, 128, 256, 16384, 2, 1), (1, 16, 64, 16, 9008, 40, 3), (2, 3, 128, 16, 16, 150, 40),
                                                                    (2, 2, 64, 32, 96, 300, 1), (4, 8, 128, 128, 1024, 16, 600), (1, 40, 128, 64, 2048, 13, 17)])
def test_a_prefix_split_over_many_and_few_ctas(nnc, kv, dtype, heads, group, d, page, shared, members, tail):
    _check(nnc, kv, dtype, [(shared, [shared + 1 + (i * 37) % tail for i in range(members)])], page, heads, group, d, scale=0.2)


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_shares_of_few_steps_that_end_one_tile_and_begin_another(nnc, kv, dtype, d):
    """Five tiles, 1 to 9 steps a share on 148 SMs: shares with fewer steps than there are stages, of two tiles each here and there."""
    for share in range(1, 10):
        for more in (0, 17):
            shared = 64 * (148 * share // 5 + more)
            _check(nnc, kv, dtype, [(shared, [shared + 1] * 40)], 64, 1, 16, d, scale=0.2)
    _check(nnc, kv, dtype, [(64 * (1 + g % 5), [64 * (1 + g % 5) + 3] * (1 + g % 3)) for g in range(160)], 64, 1, 48, d, scale=0.2)


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_tiles_of_one_sequence_s_query_heads(nnc, kv, dtype, d):
    """Every tile a sequence's 128 query heads, so queries change often; flat weights, where every row counts alike."""
    groups = [(0, []), (3175, [3176]), (1535, [1536] * 9), (720, [0, 721, 721, 718, 721]), (232, [233]), (256, [257] * 60)]
    for seed in range(8):
        _check(nnc, kv, dtype, groups, 64, 5, 128, d, seed=seed, scale=0.01)


def test_many_groups(nnc):
    for kv in (BF16, F16):
        _check(nnc, kv, kv, [(16 * (g % 9), [16 * (g % 9) + 1 + (i + g) % 30 for i in range(g % 4)]) for g in range(3, 250)], 16, 2, 4, 64)


@pytest.mark.parametrize("kv", [BF16, F16], ids=str)
def test_peaked_flat_growing_and_extreme_scores(nnc, kv):
    groups = [(640, [700, 650, 641, 640, 900, 333])]

    def change(q):
        q[0] = 0                       # all scores alike
        q[1] *= 30                     # a few positions carry everything
        q[2] *= 1e-6
        q[3, :, 0] = 300.0             # one element above the others
        return q
    for scale in (None, 0.0, -0.3, 1e-30, 4.0):
        _check(nnc, kv, kv, groups, 32, 2, 4, 64, scale=scale, change=change)
    # keys that grow with the position: the reference moves again and again
    cache, lens, starts, shared, _ = _grouped(nnc, kv, groups, 32, 1, 128, 3)
    k, v = (_randn(_gen(4), 900, 1, 128) for _ in range(2))
    k[:, 0, 0] = torch.arange(900, device="cuda") * 0.5
    held = [[], []]
    for b, n in enumerate(lens):
        first = 0 if b == 0 else 640
        if n > first:
            nnc.op_kv_write_paged(cache, k[first:n].contiguous(), v[first:n].contiguous(), _ints(range(first, n)), _ints([b] * (n - first)))
        for which, x in enumerate((k, v)):
            held[which].append(x[:n].to(kv).double().transpose(0, 1))
    q = _randn(_gen(5), len(lens), 3, 128)
    q[..., 0] = 1.0
    q = q.to(kv)
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True, scale=0.5)
    _check_attention(out, lse, q, held, lens, 0.5, 0, kv)


def test_results_are_the_ordinary_attention_s(nnc):
    """Same batch through both: they differ by the order of their sums."""
    for kv in (BF16, F16, E4M3):
        cache, lens, starts, shared, _ = _grouped(nnc, kv, [(512, [600, 513, 512, 2000]), (64, [99, 70])], 64, 4, 128, 2)
        q = _randn(_gen(3), 6, 16, 128, dtype=F16 if kv is F16 else BF16)
        out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
        want, want_lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), want_lse=True)
        # a rounding each of the result, and fp32 sums (64 steps, 2^-18)
        assert torch.allclose(out.float(), want.float(), rtol=torch.finfo(out.dtype).eps, atol=2.0 ** -12) and torch.allclose(lse, want_lse, rtol=2.0 ** -18, atol=2.0 ** -18)


def test_rows_of_wider_matrices_and_nothing_else(nnc):
    cache, lens, starts, shared, held = _grouped(nnc, BF16, [(64, [70, 64, 80]), (32, [40])], 16, 2, 128, 2)
    wide = _randn(_gen(2), 6, 3 * 4 * 128, dtype=BF16)
    q = wide[:4, 512:1024].unflatten(1, (4, 128))
    whole = torch.full((6, 1000), 9.0, dtype=BF16, device="cuda")
    out = whole[1:5, 8:520].unflatten(1, (4, 128))
    got, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), out=out, want_lse=True)
    assert got.data_ptr() == out.data_ptr()
    _check_attention(out, lse, q, held, lens, 128 ** -0.5, 0, BF16)
    keep = out.clone()
    whole[1:5, 8:520] = 9
    assert (whole == 9).all()
    same = q.contiguous()
    assert nnc.op_attn_prefix_paged(same, cache, _ints(lens), _ints(starts), _ints(shared), out=same) is same and torch.equal(same, keep)   # over its own queries
    nan_q = q.clone()
    nan_q[0, 1] = math.nan                                            # a query's NaN is its own head's
    got = nnc.op_attn_prefix_paged(nan_q, cache, _ints(lens), _ints(starts), _ints(shared))
    assert got[0, 1].isnan().all() and not got[0, [0, 2, 3]].isnan().any() and torch.equal(got[1:], keep[1:])
    assert nnc.op_attn_prefix_paged(q[:0], cache, _ints([]), _ints([0]), _ints([])).shape == (0, 4, 128)


@pytest.mark.parametrize("kv", [BF16, F16], ids=str)
def test_infinite_keys_and_values(nnc, kv):
    """An infinity among the attended values is its column's result, in the prefix or behind it; a key whose score is -infinity takes its row
    out, one of +infinity leaves no number; rows that a sequence does not attend to are its own affair."""
    groups = [(128, [150, 128, 40, 140])]
    cache, lens, starts, shared, _ = _grouped(nnc, kv, groups, 16, 1, 64, 2)
    k, v = (_randn(_gen(4), 150, 1, 64) for _ in range(2))
    v[100, 0, 3], v[20, 0, 4], v[30, 0, 5], v[35, 0, 5], v[31, 0, 6] = math.inf, -math.inf, math.inf, -math.inf, math.nan
    k[90, 0, 0] = -math.inf
    v[90] = 5.0
    tail = v.clone()
    tail[145, 0, 7], tail[135, 0, 8] = math.inf, -math.inf
    q = _randn(_gen(5), 4, 2, 64)
    q[..., 0] = 1.0
    q[3, 1, 0] = -1.0                                                 # for this one the key's score is +infinity
    q = q.to(kv)
    nnc.op_kv_write_paged(cache, k, tail, _ints(range(150)), _ints([0] * 150))
    nnc.op_kv_write_paged(cache, k[128:140].contiguous(), tail[128:140].contiguous(), _ints(range(128, 140)), _ints([3] * 12))
    out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
    assert (out[:2, :, 3] == math.inf).all() and out[2, :, 3].isfinite().all() and (out[3, 0, 3] == math.inf)
    assert (out[:3, :, 4] == -math.inf).all() and out[:, :, 5:7].isnan().all()
    assert (out[0, :, 7] == math.inf).all() and (out[0, :, 8] == -math.inf).all() and out[1:3, :, 7:9].isfinite().all()
    assert out[3, 0, 7].isfinite() and out[3, 0, 8] == -math.inf and out[3, 1].isnan().all() and lse[3, 1].isnan()
    held = [[x[:n].clone().to(kv).double().transpose(0, 1) for n in lens] for x in (k, v)]
    for b, n in enumerate(lens):                                      # the other columns are those without the row
        cols = [0, 1, 2] + list(range(9, 64))
        keep = [i for i in range(n) if i != 90]
        kk, vv = held[0][b][:, keep], held[1][b][:, keep].nan_to_num(0, 0, 0)
        o, ls = out[b:b + 1].clone(), lse[b:b + 1].clone()
        want = torch.softmax(torch.einsum("gd,nd->gn", q[b].double(), kk[0]) / 8, -1) @ vv[0]
        rows = [0] if b == 3 else [0, 1]
        # a rounding of the result and 2^-16 of the weights' sum of magnitudes (values up to 5)
        assert ((o[0].double() - want).abs()[rows][:, cols] <= torch.finfo(kv).eps / 2 * want.abs()[rows][:, cols] + 2.0 ** -13).all()
        assert (ls[0].double() - torch.logsumexp(torch.einsum("gd,nd->gn", q[b].double(), kk[0]) / 8, -1)).abs()[rows].max() < 2.0 ** -16


@pytest.mark.parametrize("kv", [BF16, F16], ids=str)
def test_shared_rows_behind_a_sequence_s_end_do_not_reach_it(nnc, kv):
    """NaN and infinities in shared rows past a shorter sequence's length, in one CTA's share and in several."""
    for shared, lens_of in ((128, [140, 40, 127, 0, 128]), (8192, [8200, 8191, 70])):
        cache, lens, starts, groups, held = _grouped(nnc, kv, [(shared, lens_of)], 16, 2, 64, 2)
        last = cache.page_table[0, shared // 16 - 1].long()
        cache.v[last, :, 15, 3], cache.v[last, :, 15, 4], cache.k[last, :, 15, 0] = math.inf, math.nan, math.nan
        q = _randn(_gen(4), len(lens), 6, 64, dtype=kv)
        out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(groups), want_lse=True)
        short = [b for b, n in enumerate(lens) if n < shared]
        _check_attention(out[short], lse[short], q[short], [[t[b] for b in short] for t in held], [lens[b] for b in short], 0.125, 0, kv)
        assert out[[b for b in range(len(lens)) if b not in short]].isnan().all()


def test_query_rows_that_overlap_and_groups_of_many_heads(nnc):
    cache, lens, starts, shared, held = _grouped(nnc, BF16, [(64, [70, 64, 80])], 16, 2, 64, 2)
    one = _randn(_gen(2), 1, 4, 64, dtype=BF16)
    out, lse = nnc.op_attn_prefix_paged(one.expand(3, 4, 64), cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
    _check_attention(out, lse, one.expand(3, 4, 64), held, lens, 0.125, 0, BF16)
    for group in (127, 128, 129):
        q = _randn(_gen(3), 3, 2 * group, 64, dtype=BF16)
        out, lse = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared), want_lse=True)
        _check_attention(out, lse, q, held, lens, 0.125, 0, BF16)


def test_pages_lengths_and_groups_out_of_range(nnc):
    cache, lens, starts, shared, held = _grouped(nnc, BF16, [(96, [100, 99]), (48, [60, 50])], 16, 2, 64, 2)
    q = _randn(_gen(2), 4, 4, 64, dtype=BF16)
    call = lambda at=lens, starts=starts, shared=shared: nnc.op_attn_prefix_paged(q, cache, _ints(at), _ints(starts), _ints(shared), want_lse=True)
    out, lse = call([2 ** 31 - 1, -3, 60, 50])                        # row 0: rows of NaN behind 100
    assert nnc.op_status() == 0x100 and (out[1] == 0).all() and (lse[1] == -math.inf).all()
    _check_attention(out[2:], lse[2:], q[2:], [t[2:] for t in held], lens[2:], 0.125, 0, BF16)
    keep = [i for i in range(100) if not 32 <= i < 48]
    page = cache.page_table[0, 2].item()
    for bad in (-1, 1 << 30):
        cache.page_table[:2, 2] = bad                                 # positions 32 .. 47 of the first group are gone
        out, lse = call()
        assert nnc.op_status() == 0x100
        _check_attention(out, lse, q, [[t[0][:, keep], t[1][:, keep[:-1]], t[2], t[3]] for t in held], [84, 83, 60, 50], 0.125, 0, BF16)
    cache.page_table[:2, 2] = page
    whole, whole_lse = call()
    assert nnc.op_status() == 0
    _check_attention(whole, whole_lse, q, held, lens, 0.125, 0, BF16)
    # groups that leave the batch or descend: no address leaves its range, sequences of no group attend alone
    for wrong in ([0, 2, 9], [-5, 2, 4]):
        out, lse = call(starts=wrong)
        assert nnc.op_status() == 0x100
        _check_attention(out, lse, q, held, lens, 0.125, 0, BF16)
    for wrong in ([3, 1, 4], [4, 4, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        call(starts=wrong)
        assert nnc.op_status() == 0x100
    out, lse = call(starts=[1, 2, 3])                                 # the first and the last sequence alone
    assert nnc.op_status() == 0
    _check_attention(out, lse, q, held, lens, 0.125, 0, BF16)
    out, lse = call(shared=[-7, 48])
    assert nnc.op_status() == 0x100
    _check_attention(out, lse, q, held, lens, 0.125, 0, BF16)
    call(shared=[2 ** 31 - 1, 2 ** 31 - 1])                           # the whole table: entries of -1 and rows of NaN among it
    assert nnc.op_status() == 0x100


def test_16_bit_results_of_long_prefixes_are_rounded_once(nnc):
    """65536 positions in few shares: the tensor cores' sums, two terms of the weights and the rounding, against 64 bits: the error's
    root mean square is within a tenth of the rounding's own (eps / 2 / sqrt(3) of values spread over a binade: at most)."""
    for kv in (BF16, F16):
        n, members = 65536, 4
        cache, lens, starts, shared, held = _grouped(nnc, kv, [(n, [n + 1] * members)], 256, 1, 128, 5)
        q = _randn(_gen(6), members, 128 // members * 12, 128, dtype=kv)
        out = nnc.op_attn_prefix_paged(q, cache, _ints(lens), _ints(starts), _ints(shared))
        for b in range(members):
            want = torch.softmax(torch.einsum("gd,nd->gn", q[b].double(), held[0][b][0]) * 128 ** -0.5, -1) @ held[1][b][0]
            error, rounding = (out[b].double() - want).norm(), (want.to(kv).double() - want).norm()
            assert error < 1.1 * rounding, (kv, b, (error / rounding).item())


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_a_captured_step_behind_a_prefix(nnc, kv):
    """Append and attend: captured once, replayed while lengths move on and a sequence changes its group; beside it the same on a stream
    of its own with a scratch of its own."""
    heads, group, d, page, steps = 2, 4, 128, 16, 24
    groups = [(320, [321, 350, 330]), (64, [64, 90])]
    sides = []
    for side in range(2):
        cache, lens, starts, shared, held = _grouped(nnc, kv, [(p, [n + steps for n in of]) for p, of in groups], page, heads, d, 7 + side)
        start = [n - steps for n in lens]
        g = _gen(9)
        new_k, new_v, new_q = (_randn(g, steps, len(lens), x, d, dtype=BF16) for x in (heads, heads, heads * group))
        hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
        for which, new in enumerate((new_k, new_v)):
            for b, n in enumerate(start):
                held[which][b][:, n:n + steps] = hold(new[:, b]).transpose(0, 1)
        at = [_ints(start), _ints(start), _ints(starts), _ints(shared)]
        buffers = [torch.zeros(len(lens), x, d, dtype=BF16, device="cuda") for x in (heads, heads, heads * group)]
        own = nnc.attn_prefix_scratch(len(lens), heads * group, d)

        def step(cache=cache, at=at, buffers=buffers, own=own):
            nnc.op_kv_write_paged(cache, buffers[0], buffers[1], at[0])
            at[1].copy_(at[0] + 1)
            out, lse = nnc.op_attn_prefix_paged(buffers[2], cache, at[1], at[2], at[3], scratch=own, want_lse=True)
            at[0].add_(1)
            return out, lse

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
            at[0].copy_(_ints(start))
            graph = torch.cuda.CUDAGraph()
            stream.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                results = step()
        sides.append((graph, stream, buffers, at, (new_k, new_v, new_q), results, held, start, step))
    for i in range(steps):
        for graph, stream, buffers, at, news, *_ in sides:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for t, new in zip(buffers, news):
                    t.copy_(new[i])
                if i == steps // 2:                                       # the first group ends a sequence earlier
                    at[2].copy_(_ints([0, 2, 5]))
                    at[3].copy_(_ints([320, 0]))
                graph.replay()
        torch.cuda.synchronize()
        for _, _, buffers, _, _, (out, lse), held, start, _ in sides:
            now = [n + i + 1 for n in start]
            _check_attention(out, lse, buffers[2], [[t[:, :n] for t, n in zip(x, now)] for x in held], now, d ** -0.5, 0, kv)
    assert nnc.op_status() == 0


def test_refusals_of_the_binding(nnc):
    cache, lens, starts, shared, _ = _grouped(nnc, BF16, [(32, [40, 40])], 16, 2, 64, 1)
    q, lens, starts, shared = _randn(_gen(1), 2, 4, 64, dtype=BF16), _ints(lens), _ints(starts), _ints(shared)
    call = lambda q=q, lens=lens, starts=starts, shared=shared, **kw: nnc.op_attn_prefix_paged(q, cache, lens, starts, shared, **kw)
    scratch = nnc.attn_prefix_scratch(2, 4, 64)
    for refused in (lambda: call(q=q[..., :32]), lambda: call(q=q.cpu()), lambda: call(lens=lens[:1]), lambda: call(starts=starts[:1]), lambda: call(starts=starts.long()),
                    lambda: call(shared=shared[:0], starts=starts[:1]), lambda: call(shared=_ints([1, 2, 3]), starts=_ints([0, 1, 1, 2])), lambda: call(shared=shared.cpu()),
                    lambda: call(out=q[:, :2]), lambda: call(out=cache.k.view(-1)[:q.numel()].view_as(q)), lambda: call(scratch=scratch.cpu()),
                    lambda: call(out=q.clone().requires_grad_()), lambda: nnc.attn_prefix_scratch(2, 4, 96), lambda: nnc.attn_prefix_scratch(-1, 4, 64)):
        with pytest.raises(ValueError):
            refused()
    for refused, status in ((lambda: call(scratch=scratch[:-256]), -2), (lambda: call(q=q.half()), -1)):
        with pytest.raises(nnc.NncError) as e:
            refused()
        assert e.value.status == status
    assert torch.equal(call(scratch=nnc.attn_prefix_scratch(9, 4, 64)), call())      # a larger one will do


@pytest.mark.parametrize("kv", [BF16, F16], ids=str)
@pytest.mark.parametrize("heads,group,d,page,shared,members", [(2, 12, 64, 128, 65536, 48), (1, 128, 64, 64, 20000, 7), (4, 30, 128, 32, 9000, 25), (8, 1, 64, 16, 8192, 130)])
def test_long_shares_of_several_tiles(nnc, kv, heads, group, d, page, shared, members):
    """Dozens of steps a CTA, its share beginning and ending inside tiles: every ring wraps many times over."""
    _check(nnc, kv, kv, [(shared, [shared // page * page + 1 + 3 * i for i in range(members)])], page, heads, group, d)
