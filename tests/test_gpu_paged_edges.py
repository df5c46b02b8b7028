"""Attention over the paged cache where its operands leave the ordinary: rows of zeros, scales at the ends of their range,
infinities, long shares.  Plain 64-bit forms and bounds as in test_gpu_paged."""
import math

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F16, F32, _check_attention, _fill, _gen, _ints, _paged, _randn, nnc, quantise64, scratch  # noqa: F401

pytestmark = pytest.mark.gpu


def _held(k, v):
    """What an E4M3 cache holds of rows [n][heads][d] of one sequence."""
    return [[quantise64(x)[0].transpose(0, 1)] for x in (k, v)]


# ---- the sum of the weights ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("n", [200, 8193])
def test_a_row_of_large_values_leaves_the_sum_of_the_weights_alone(nnc, scratch, dtype, n):
    """One value row with the scale 2^60, the others with 2^-60, its score above or below theirs: the sum counts every row by its own
    weight, whatever its values' scale.  Many sequences of the same pages, so that a CTA holds whole ones."""
    g = _gen(n)
    d, heads, group, page, batch = 64, 1, 2, 64, 500
    q = _randn(g, batch, heads * group, d).to(dtype)
    q[:, :, 0] = 3.0
    k, v = (_randn(g, n, heads, d) for _ in range(2))
    k[:, :, 0] = 0
    v *= 2.0 ** -53
    v[n // 3] = 448 * 2.0 ** 60
    pages = -(-n // page)
    cache = nnc.PagedKV.empty(pages, page, heads, d, E4M3, batch, pages)
    cache.page_table[:] = torch.arange(pages, device="cuda", dtype=torch.int32)
    lens = [n] * batch
    for above in (16.0, 14.2, 0.0, -14.2, -40.0):
        k[n // 3, :, 0] = above / 3.0 / d ** -0.5
        nnc.op_kv_write_paged(cache, k, v, _ints(range(n)), _ints([0] * n))
        out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
        _check_attention(out, lse, q, [t * batch for t in _held(k, v)], lens, d ** -0.5, 0, E4M3)


# ---- rows of zeros ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-5, 1e-7, 1e-10])
@pytest.mark.parametrize("n,d,group", [(513, 64, 3), (70, 128, 1), (5000, 128, 16)])
def test_value_rows_of_zeros_take_no_bits_from_the_others(nnc, scratch, dtype, size, n, d, group):
    """Rows of zeros, written or never written, at scores up to 14 above the others: their codes are 0 and weigh nothing in the
    result, so its accuracy is the other rows'."""
    g = _gen(n + group)
    heads = 2
    q = _randn(g, 3, heads * group, d)
    q[:, :, 0] = 3.0
    k, v = (_randn(g, n, heads, d) for _ in range(2))
    v *= size
    k[:, :, 0] = 0
    for row, above in ((0, 14.0), (n // 2, 10.0), (n - 2, 0.0), (n - 1, -3.0)):
        v[row] = 0
        k[row, :, 0] = above / 3.0 / d ** -0.5
    cache = _paged(nnc, E4M3, [n, n, 40], 32, heads, d, 1)
    for b in range(2):
        nnc.op_kv_write_paged(cache, k, v, _ints(range(n)), _ints([b] * n))
    table = cache.page_table[2, :2].long()
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):       # the third sequence: as PagedKV.empty leaves it
        pool.view(torch.uint8)[table], scale[table] = 0, 127
    nnc.op_kv_write_paged(cache, k[:7], v[:7], _ints(range(7)), _ints([2] * 7))
    held = _held(k, v)
    zeros = torch.zeros(heads, 33, d, device="cuda").double()
    held = [t * 2 + [torch.cat([t[0][:, :7], zeros], 1)] for t in held]
    out, lse = nnc.op_attn_decode_paged(q.to(dtype), cache, _ints([n, n, 40]), scratch=scratch, want_lse=True)
    _check_attention(out, lse, q.to(dtype), held, [n, n, 40], d ** -0.5, 0, E4M3)
    nothing, _ = nnc.op_attn_decode_paged(q.to(dtype), cache, _ints([1, 1, 0]), scratch=scratch, want_lse=True)
    assert (nothing == 0).all()                                                     # nothing but a row of zeros


# ---- infinities ------------------------------------------------------------------------------------------------------

def _drop(held, gone):
    n = held[0][0].shape[1]
    keep = [i for i in range(n) if i not in gone]
    return [[t[0][:, keep]] for t in held], n - len(gone)


@pytest.mark.parametrize("kv,dtype", [(BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)], ids=str)
@pytest.mark.parametrize("n", [40, 3001])
def test_infinite_keys_take_their_rows_out_or_decide(nnc, scratch, kv, dtype, n):
    """A score of -infinity weighs nothing; one of +infinity leaves no number."""
    g = _gen(n)
    d, heads, group = 128, 2, 4
    q = _randn(g, 1, heads * group, d, dtype=dtype)
    q[0, :, 5] = torch.tensor([-1.3, -0.7, 1.1, -2.9] * heads, device="cuda", dtype=dtype)    # head 2 of each group meets +infinity
    k, v = (_randn(g, n, heads, d, dtype=kv) for _ in range(2))
    rows = [3, n // 2, n - 1]
    for r in rows:
        k[r, :, 5] = math.inf
    cache = _paged(nnc, kv, [n], 16, heads, d, 1)
    nnc.op_kv_write_paged(cache, k, v, _ints(range(n)), _ints([0] * n))
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints([n]), scratch=scratch, want_lse=True)
    decided = [2, 6]
    others = [0, 1, 3, 4, 5, 7]
    assert out[0, decided].isnan().all()
    held, left = _drop([[t.double().transpose(0, 1)] for t in (k, v)], rows)
    split = lambda t: t.unflatten(1, (heads, group))[:, :, [0, 1, 3]].flatten(1, 2)
    _check_attention(split(out), split(lse[..., None])[..., 0], split(q), held, [left], d ** -0.5, 0, kv)
    assert lse[0, others].isfinite().all()


@pytest.mark.parametrize("kv,dtype", [(BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)], ids=str)
@pytest.mark.parametrize("n,d,group,window", [(1, 64, 1, 0), (40, 128, 4, 0), (40, 128, 4, 30), (700, 64, 12, 0), (30011, 128, 5, 0), (9000, 64, 17, 8100)])
@pytest.mark.parametrize("spread", [1.0, 12.0])
def test_infinite_values_are_what_a_weighted_sum_makes_of_them(nnc, scratch, kv, dtype, n, d, group, window, spread):
    """Every attended weight is positive, however small: one infinity in a column of values is the column's result, two of
    different signs and NaN leave no number, the other columns are finite."""
    g = _gen(n + d)
    heads = 2
    q = (_randn(g, 2, heads * group, d) * spread).to(dtype)
    k, v = (_randn(g, n, heads, d, dtype=kv) for _ in range(2))
    first = max(0, n - window) if window else 0
    at = lambda f: first + int((n - 1 - first) * f)
    for f, column, x in ((0.0, 1, math.inf), (0.31, 2, -math.inf), (0.5, 9, math.inf), (0.9, 9, math.inf), (0.2, 33, math.inf), (0.7, 33, -math.inf),
                         (0.4, 40, math.nan), (0.6, 41, math.inf), (0.61, 41, math.nan), (1.0, 63, -math.inf), (0.77, d - 2, math.inf)):
        v[at(f), 1 if column == 9 else slice(None), column] = x
    cache = _paged(nnc, kv, [n, n], 64, heads, d, 1)
    for b in range(2):
        nnc.op_kv_write_paged(cache, k, v, _ints(range(n)), _ints([b] * n))
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints([n, n]), window=window, scratch=scratch, want_lse=True)
    seen = v[first:].double()
    plus, minus, nan = (seen == math.inf).any(0), (seen == -math.inf).any(0), seen.isnan().any(0)         # [heads][d]
    lost, up, down = nan | (plus & minus), plus & ~minus & ~nan, minus & ~plus & ~nan
    got = out.unflatten(1, (heads, group))
    for mask, test in ((lost, got.isnan()), (up, got == math.inf), (down, got == -math.inf)):
        mask = mask[None, :, None].expand_as(got)
        assert test[mask].all() and not test[~mask].any()
    # the finite columns, against the values without the others
    clean = torch.where((plus | minus | nan)[None], 0.0, v.nan_to_num(0.0, 0.0, 0.0).double())
    held = [[x.double().transpose(0, 1)] * 2 for x in (k, clean)]
    finite = torch.where((plus | minus | nan)[None, :, None].expand_as(got), torch.zeros((), dtype=out.dtype, device="cuda"), got).flatten(1, 2)
    _check_attention(finite, lse, q, held, [n, n], d ** -0.5, window, kv)


# ---- long shares -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv,dtype", [(F16, F16), (BF16, BF16), (E4M3, F16), (E4M3, BF16)], ids=str)
def test_16_bit_results_of_a_share_of_131072_positions_carry_no_drift(nnc, scratch, kv, dtype):
    """600 sequences that share one run of pages, so that a CTA sums up whole sequences: the mean distance of all results from the
    rounded exact ones, which shows sums that are cut at every addition."""
    n, d, batch = 131072, 64, 600
    g = _gen(5)
    k, v = _randn(g, n, 1, d) * 0.5, _randn(g, n, 1, d).abs() + 0.5                 # sums of one sign
    pages = n // 256
    cache = nnc.PagedKV.empty(pages, 256, 1, d, kv, batch, pages)
    cache.page_table[:] = torch.arange(pages, device="cuda", dtype=torch.int32)
    nnc.op_kv_write_paged(cache, k, v, _ints(range(n)), torch.zeros(n, dtype=torch.int32, device="cuda"))
    q = _randn(g, batch, 1, d, dtype=dtype)
    out = nnc.op_attn_decode_paged(q, cache, torch.full((batch,), n, dtype=torch.int32, device="cuda"), scratch=scratch)
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    k64, v64 = hold(k)[:, 0], hold(v)[:, 0]
    want = torch.softmax(q[:, 0].double() @ k64.T * d ** -0.5, -1) @ v64
    off = ((out[:, 0].double() - want.to(dtype).double()) / want).mean().item()
    # Against the exact values themselves the mean would be the inputs' rounding: the results of one column lie closer together than a
    # step of bf16.  Against the rounded ones, an error moves as many results by a whole step as make it up in the mean.  Of 38400
    # results, each off by at most half a step either way, the mean has a spread of at most eps / 2 / sqrt(3 * 38400), of which five are
    # allowed.  Cuts inside one block's sum (64 positions a warp, two or three terms: 12 additions at 2^-23) and the weights'
    # own rounding (2^-21) are systematic at most.
    allowed = 5 * torch.finfo(dtype).eps / 2 / math.sqrt(3 * batch * d) + 12 * 2.0 ** -23 + 2.0 ** -21
    assert abs(off) <= allowed, (off, allowed)


# ---- what 16-bit results lose ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)], ids=str)
def test_16_bit_results_are_rounded_once(nnc, scratch, kv, dtype):
    """Two positions with exact scores: a result is the exact one's rounding, unless that lies within fp32's errors of a tie."""
    batch, heads, group, d = 512, 4, 4, 64
    g = _gen(31)
    q, k = torch.zeros(batch, heads * group, d, device="cuda"), torch.zeros(2 * batch, heads, d, device="cuda")
    q[..., 0], k[..., 0] = _randn(g, batch, heads * group), _randn(g, 2 * batch, heads).clamp(-2, 2)
    q, v = q.clamp(-4, 4).to(dtype), _randn(g, 2 * batch, heads, d)
    cache = nnc.PagedKV.empty(batch, 16, heads, d, kv, batch, 1)
    cache.page_table[:, 0] = torch.arange(batch, device="cuda", dtype=torch.int32)
    seq, pos = _ints([b for b in range(batch) for _ in range(2)]), _ints([0, 1] * batch)
    nnc.op_kv_write_paged(cache, k, v, pos, seq)
    out = nnc.op_attn_decode_paged(q, cache, _ints([2] * batch), scale=0.125, scratch=scratch)
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    k64, v64 = (hold(x).view(batch, 2, heads, d) for x in (k, v))
    score = 0.125 * torch.einsum("bhgd,bnhd->bhgn", q.double().view(batch, heads, group, d), k64)
    p = torch.softmax(score, -1)
    want, size = (torch.einsum("bhgn,bnhd->bhgd", p, x).reshape(out.shape) for x in (v64, v64.abs()))
    step = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -14 if dtype is F16 else 2.0 ** -126)))) * torch.finfo(dtype).eps
    # fp32 part, of sum p |v|: scores of at most 1.5 binary digits, from exact products (2^-23 of a weight), exp2 (2^-22) and the same in
    # the other weight, the weights' terms (2^-22), sum, reciprocal and products (five times 2^-24): below 2^-20
    off = (out.double() - want).abs() - step / 2 - 2.0 ** -20 * size
    assert (off <= 0).all(), ((off > 0).sum().item(), (off / step).max().item())


# ---- the binding -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("lens", [[5], [4097], [30011, 0, 70000]])
def test_a_call_without_scratch_clears_the_tickets_of_its_own(nnc, scratch, lens):
    """The scratch that such a call makes may be memory that held anything, and only its first bytes are cleared."""
    cache = _paged(nnc, BF16, lens, 64, 2, 128, 1, nan=False)
    _fill(nnc, cache, lens, 1)
    q = _randn(_gen(3), len(lens), 8, 128, dtype=BF16)
    want = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    for _ in range(3):
        used = [torch.full((16 << 20,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(3)]
        at = {t.data_ptr() for t in used}
        del used
        got = nnc.op_attn_decode_paged(q, cache, _ints(lens), want_lse=True)
        own = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")      # the freed scratch again: what the call left
        assert own.data_ptr() in at and not own[:8192].any()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if lens == [5]:                                                     # one CTA per head: nothing is split, nothing else written
            assert (own[8192:] == 0xff).all()
        del own


def test_outputs_that_overlap_what_a_call_reads_are_refused(nnc, scratch):
    """Exactly those: parts of one buffer that have no element in common are as good as two buffers."""
    freq, _ = nnc.rope_frequencies(64)
    pos = _ints([3, 5, 7, 9])
    buf = torch.zeros(20000, dtype=BF16, device="cuda")
    rows = lambda at, row, head: torch.as_strided(buf, (4, 3, 64), (row, head, 1), at)
    touches = lambda a, b: bool(set(_elements(a)) & set(_elements(b)))
    _elements = lambda t: torch.arange(20000).as_strided(t.shape, t.stride(), t.storage_offset()).flatten().tolist()
    g = torch.Generator().manual_seed(2)
    kinds = [(192, 64), (64, 256), (1000, 72), (384, 128), (400, 128), (72, 1000), (200, 64), (1, 64 * 8), (64, 0)]
    seen = set()
    for _ in range(400):
        (rx, hx), (ry, hy) = (kinds[int(torch.randint(len(kinds) if i == 0 else len(kinds) - 2, (1,), generator=g))] for i in range(2))
        ax, ay = (int(torch.randint(0, 600, (1,), generator=g)) for _ in range(2))
        x, y = rows(ax, rx, hx), rows(ay, ry, hy)
        if x.data_ptr() == y.data_ptr() and x.stride() == y.stride():
            continue
        seen.add(touches(x, y))
        if touches(x, y):
            with pytest.raises(ValueError, match="no part of"):
                nnc.op_rope(x, pos, freq, out=y)
        else:
            assert nnc.op_rope(x, pos, freq, out=y) is y
    assert seen == {False, True}
    fused = torch.zeros(5, 12, 64, dtype=BF16, device="cuda")                       # heads of one projection, next to one another
    five = _ints([0] * 5)
    nnc.op_rope(fused[:, :4], five, freq, out=fused[:, 4:8])
    nnc.op_rope(fused[:, :4], five, freq, out=fused[:, :4])
    for out in (fused[:, 3:7], fused[:, 1:5]):
        with pytest.raises(ValueError):
            nnc.op_rope(fused[:, :4], five, freq, out=out)
    nnc.op_rope(fused[:1, :4], five[:1], freq, out=fused[1:2, :4])
    # the cache's operations
    cache = _paged(nnc, BF16, [40], 16, 2, 64, 1)
    held = _fill(nnc, cache, [40], 1)
    three, zero = _ints([1, 2, 30]), _ints([0, 0, 0])
    pair = torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    nnc.op_kv_read_paged(cache, three, zero, out=(pair[:, :2], pair[:, 2:]))
    pool = cache.k.flatten(0, 2)[:6].view(3, 2, 64)
    for out in ((pair[:, :2], pair[:, :2]), (pair[:, :2], pair[:, 1:3]), (None, pair[:, :2]), (pair[:, :2], pool), (pool, pair[:, :2])):
        with pytest.raises(ValueError):
            nnc.op_kv_read_paged(cache, three, zero, out=out)
    with pytest.raises(ValueError):
        nnc.op_kv_write_paged(cache, pool, torch.zeros_like(pool), three, zero)
    # attention: q itself is allowed, its neighbours are not
    q = _randn(_gen(4), 1, 8, 64, dtype=BF16)
    want = nnc.op_attn_decode_paged(q, cache, _ints([40]), scratch=scratch)
    wide = torch.zeros(1, 16, 64, dtype=BF16, device="cuda")
    wide[:, 2:10] = q
    with pytest.raises(ValueError):
        nnc.op_attn_decode_paged(wide[:, 2:10], cache, _ints([40]), scratch=scratch, out=wide[:, 4:12])
    nnc.op_attn_decode_paged(wide[:, 2:10], cache, _ints([40]), scratch=scratch, out=wide[:, 2:10])
    assert torch.equal(wide[:, 2:10], want) and not wide[:, :2].any() and not wide[:, 10:].any()


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (E4M3, F32)], ids=str)
@pytest.mark.parametrize("heads,group", [(2, 4), (1, 16), (1, 40)])
def test_attention_over_its_own_queries(nnc, scratch, kv, dtype, heads, group):
    lens = [30000, 0, 17, 9000]
    cache = _paged(nnc, kv, lens, 64, heads, 128, 1)
    _fill(nnc, cache, lens, 1)
    q = _randn(_gen(3), len(lens), heads * group, 128, dtype=dtype)
    want, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    for _ in range(5):
        own = q.clone()
        got, again = nnc.op_attn_decode_paged(own, cache, _ints(lens), scratch=scratch, out=own, want_lse=True)
        assert got is own or got.data_ptr() == own.data_ptr()
        assert torch.equal(own, want) and torch.equal(lse, again)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_gradients_flow_through_the_rotation(nnc, interleaved, dtype):
    """x + R x, a step further through autograd: the gradient is g + R^T g, the second derivative of a quadratic the product of both."""
    g = _gen(8)
    freq, _ = nnc.rope_frequencies(48, 1e4)
    pos = _ints([2, 1000, 70001, 5])
    rope = lambda t, **kw: nnc.op_rope(t, pos, freq, interleaved=interleaved, amplitude=1.5, **kw)
    x, up = (_randn(g, 4, 3, 80, dtype=dtype) for _ in range(2))
    leaf = x.clone().requires_grad_()
    y = rope(leaf)
    assert y.requires_grad and torch.equal(y.detach(), rope(x))
    y.backward(up)
    assert torch.equal(leaf.grad, rope(up, inverse=True))
    leaf.grad = None
    rope(leaf).sum().backward()                                       # an expanded gradient
    assert torch.equal(leaf.grad, rope(torch.ones_like(x), inverse=True))
    part = torch.zeros(4, 5, 80, dtype=dtype, device="cuda", requires_grad=True)       # some heads of a fused projection, not contiguous
    rope(part[:, 1:4], inverse=True).backward(up)
    assert torch.equal(part.grad[:, 1:4], rope(up)) and not part.grad[:, [0, 4]].any()
    first, = torch.autograd.grad(rope(leaf), leaf, up.requires_grad_(), create_graph=True)
    second, = torch.autograd.grad(first, up, x)
    assert torch.equal(second, rope(x))
    with torch.no_grad():
        assert not rope(leaf).requires_grad
    for out in (torch.empty_like(x), leaf):
        with pytest.raises(ValueError):
            rope(leaf, out=out)
    with pytest.raises(ValueError):
        rope(x, out=leaf)
    with torch.no_grad():
        rope(x, out=leaf)


def test_gradients_notice_what_changed_before_them(nnc, scratch):
    freq, _ = nnc.rope_frequencies(64)
    pos = _ints([4])
    leaf = torch.ones(1, 1, 64, device="cuda", requires_grad=True)
    y = nnc.op_rope(leaf, pos, freq)
    pos += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    kept = torch.ones(1, 1, 64, dtype=BF16, device="cuda")
    cache = _paged(nnc, BF16, [1], 16, 1, 64, 1)
    _fill(nnc, cache, [1], 1)
    for overwrite in (lambda t: nnc.op_rope(t, pos, freq, out=t), lambda t: nnc.op_attn_decode_paged(t, cache, _ints([1]), scratch=scratch, out=t),
                      lambda t: nnc.op_kv_read_paged(cache, _ints([0]), out=(t, torch.empty_like(t))),
                      lambda t: nnc.op_kv_read_paged(cache, _ints([0]), out=(torch.empty_like(t), t))):
        weight = torch.ones(1, 1, 64, dtype=BF16, device="cuda", requires_grad=True)
        y = weight * kept                                             # keeps `kept` for the gradient
        overwrite(kept)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    with torch.inference_mode():
        t = torch.ones(1, 1, 64, dtype=BF16, device="cuda")
        nnc.op_rope(t, pos, freq, out=t)
