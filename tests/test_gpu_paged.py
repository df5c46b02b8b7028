"""Rotary positions and the paged key-value cache against plain 64-bit forms of the same operations, at the sizes, strides
and masks where they can go wrong.

Bounds: a result of type t is off by half a step of t, eps(t) / 2 of its value, for the one rounding at the end, plus what
fp32 arithmetic before it leaves; each test says what that is made of."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_b200 import binding
    return binding


@pytest.fixture(scope="module")
def scratch(nnc):
    return nnc.attn_paged_scratch()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- rotary positions ------------------------------------------------------------------------------------------------

def rope64(x, pos, freq, interleaved=False, amplitude=1.0, inverse=False):
    rot = 2 * freq.numel()
    angle = (pos.double()[:, None] * freq)[:, None] * (-1 if inverse else 1)
    c, s = torch.cos(angle), torch.sin(angle)
    x = x.double().clone()
    a, b = (x[..., 0:rot:2].clone(), x[..., 1:rot:2].clone()) if interleaved else (x[..., :rot // 2].clone(), x[..., rot // 2:rot].clone())
    ya, yb = amplitude * (a * c - b * s), amplitude * (b * c + a * s)
    size = torch.zeros_like(x)
    if interleaved:
        x[..., 0:rot:2], x[..., 1:rot:2] = ya, yb
        size[..., 0:rot:2] = size[..., 1:rot:2] = amplitude * (a.abs() + b.abs())
    else:
        x[..., :rot // 2], x[..., rot // 2:rot] = ya, yb
        size[..., :rot // 2] = size[..., rot // 2:rot] = amplitude * (a.abs() + b.abs())
    return x, size


def _check_rope(y, x, pos, freq, **kw):
    # fp32 part, relative to |a| + |b|: the angle (2^-28 turns: 2^-25), sine and cosine (2 units: 2^-23), the products and
    # the sum (2^-24 each), the amplitude's product (2^-24): under 2^-21 together
    want, size = rope64(x, pos, freq, **kw)
    tol = torch.finfo(y.dtype).eps / 2 * want.abs() + 2.0 ** -21 * size + (torch.finfo(y.dtype).smallest_normal if y.dtype is F16 else 0) * 2.0 ** -10
    rest = size == 0
    bad = ((y.double() - want).abs() > tol)
    assert not bad.any(), (bad.sum().item(), (y.double() - want).abs().max().item())
    untouched = 2 * freq.numel()
    assert torch.equal(y[..., untouched:], x[..., untouched:].to(y.dtype)) and rest is not None


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,d,rot", [(1, 1, 64, 64), (1, 40, 128, 128), (3, 5, 80, 20), (7, 3, 96, 48), (5, 2, 66, 66), (2, 3, 9, 2),
                                                (33, 1, 256, 128), (17, 70, 192, 64), (301, 2, 128, 32), (2, 2, 1024, 1024),
                                                (5, 3, 96, 24), (7, 2, 84, 40), (1801, 33, 128, 128), (2003, 24, 96, 48), (1999, 40, 80, 20),
                                                (2500, 30, 96, 24), (40001, 1, 64, 64), (9001, 3, 40, 8)])
def test_rope(nnc, dtype, interleaved, tokens, heads, d, rot):
    g = _gen(tokens * 1000 + d)
    x = _randn(g, tokens, heads, d, dtype=dtype)
    pos = torch.randint(-50000, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    freq, _ = nnc.rope_frequencies(rot, 1e4)
    keep = x.clone()
    for inverse in (False, True):
        y = nnc.op_rope(x, pos, freq, interleaved=interleaved, amplitude=1.25, inverse=inverse)
        _check_rope(y, x, pos, freq, interleaved=interleaved, amplitude=1.25, inverse=inverse)
    assert torch.equal(x, keep)
    z = x.clone()
    assert nnc.op_rope(z, pos, freq, interleaved=interleaved, amplitude=1.25, out=z) is z     # in place
    assert torch.equal(z, nnc.op_rope(x, pos, freq, interleaved=interleaved, amplitude=1.25))


def test_rope_at_the_ends_of_the_position_range(nnc):
    pos = _ints([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1 << 30])
    freq, _ = nnc.rope_frequencies(128, 1e6)
    x = _randn(_gen(3), 7, 4, 128)
    _check_rope(nnc.op_rope(x, pos, freq), x, pos, freq)
    assert torch.equal(nnc.op_rope(x, pos, freq)[0], x[0])
    # quarter turns are exact up to fp32: no angle near one is cut to 32 bits before it is reduced
    quarter = torch.full((64,), math.pi / 2, dtype=torch.float64, device="cuda")
    y = nnc.op_rope(x, _ints([4 * 10 ** 8 + i for i in range(7)]), quarter)
    want, _ = rope64(x, torch.tensor([i % 4 for i in range(7)], device="cuda"), quarter)
    # pi / 2 itself is off by 6.1e-17 in 64 bits: 4e8 of it is 2.5e-8, beside the bound above
    assert (y.double() - want).abs().max() < 2.0 ** -20 * x.abs().max()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=str)
def test_rope_strides(nnc, dtype):
    g = _gen(4)
    freq, amp = nnc.rope_frequencies(64, 1e6, "ramp_index", 8.0, 4096.0, 1.0, 32.0)
    fused = _randn(g, 6, 12, 128, dtype=dtype)                     # query, key and value heads of one projection
    pos = _ints([0, 9, 3, 77, 5, 4095])
    before = fused.clone()
    part = fused[:, :10]
    y = nnc.op_rope(part, pos, freq, amplitude=amp)
    _check_rope(y, part, pos, freq, amplitude=amp)
    nnc.op_rope(part, pos, freq, amplitude=amp, out=part)
    assert torch.equal(part, y) and torch.equal(fused[:, 10:], before[:, 10:])
    major = _randn(g, 10, 6, 128, dtype=dtype).transpose(0, 1)     # head-major
    _check_rope(nnc.op_rope(major, pos, freq), major, pos, freq)
    odd = _randn(g, 6, 10, 131, dtype=dtype)[..., 1:129]           # no 16-byte rows
    _check_rope(nnc.op_rope(odd, pos, freq, interleaved=True), odd, pos, freq, interleaved=True)
    one = _randn(g, 1, 10, 128, dtype=dtype).expand(6, 10, 128)    # one row turned by many positions
    _check_rope(nnc.op_rope(one, pos, freq), one, pos, freq)
    wide = torch.full((6, 10, 200), 7.0, dtype=dtype, device="cuda")
    nnc.op_rope(part, pos, freq, out=wide[..., 8:136])
    assert (wide[..., :8] == 7).all() and (wide[..., 136:] == 7).all()
    with pytest.raises(ValueError):
        nnc.op_rope(part, pos, freq, out=torch.empty(1, 10, 128, dtype=dtype, device="cuda").expand(6, 10, 128))
    assert nnc.op_rope(part[:0], pos[:0], freq).shape == (0, 10, 128)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_inverse_is_the_gradient(nnc, interleaved):
    g = _gen(5)
    freq, _ = nnc.rope_frequencies(24, 1e4)
    x, up = _randn(g, 3, 2, 40), _randn(g, 3, 2, 40)
    pos = _ints([2, 1000, 70001])
    f = lambda t: (nnc.op_rope(t, pos, freq, interleaved=interleaved, amplitude=1.5).double() * up.double()).sum().item()
    grad = nnc.op_rope(up, pos, freq, interleaved=interleaved, amplitude=1.5, inverse=True)
    leaf = x.double().requires_grad_()
    a64 = (pos.double()[:, None] * freq)[:, None]
    rot = 24
    a, b = (leaf[..., 0:rot:2], leaf[..., 1:rot:2]) if interleaved else (leaf[..., :12], leaf[..., 12:rot])
    ya, yb = 1.5 * (a * a64.cos() - b * a64.sin()), 1.5 * (b * a64.cos() + a * a64.sin())
    turned = torch.stack([ya, yb], -1).flatten(-2) if interleaved else torch.cat([ya, yb], -1)
    (torch.cat([turned, leaf[..., rot:]], -1) * up.double()).sum().backward()
    assert (grad.double() - leaf.grad).abs().max() < 2.0 ** -20 * 3 * up.abs().max()
    for at in ((0, 0, 0), (1, 1, 13), (2, 0, 23), (2, 1, 39)):
        step = torch.zeros_like(x)
        step[at] = 1.0     # the operator is linear: any step will do
        # fp32 outputs of size ~5 are off by 2^-21 of it each; two of them change by the step
        assert abs((f(x + step) - f(x - step)) / 2 - grad[at].item()) < 80 * 2.0 ** -20


# ---- rows of the cache -----------------------------------------------------------------------------------------------

def power64(e):
    """2^e for whole e, from its bits: torch.ldexp multiplies by pow(2, e), which may be off in the last place."""
    return (e.long() + 1023 << 52).view(torch.float64)


def quantise64(x):
    """Values that a row becomes in E4M3 with its power-of-two scale (finite rows), and the exponents."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -60)
    for step in range(-60, 60):
        e = torch.where(top > 448 * 2.0 ** step, step + 1.0, e)
    e = torch.where(top > 0, e, 0.0)
    y = x * power64(-e)
    unit = power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / unit) * unit).clamp(-448, 448) * power64(e), e[..., 0]


def _paged(nnc, dtype, lens, page, heads, d, seed, spare=2, nan=True):
    """A cache laid out for sequences of the given lengths, pages in no order; unused bytes are NaN (or NaN codes)."""
    used = [-(-n // page) for n in lens]
    cache = nnc.PagedKV.empty(sum(used) + spare, page, heads, d, dtype, len(lens), max(used + [1]))
    g = torch.Generator()
    g.manual_seed(seed)
    order = torch.randperm(sum(used) + spare, generator=g).int()
    at = 0
    for b, n in enumerate(used):
        cache.page_table[b, :n] = order[at:at + n]
        at += n
    if nan:
        for pool in (cache.k, cache.v):
            pool.view(torch.uint8).fill_(0x7f) if dtype is E4M3 else pool.fill_(math.nan)
    return cache


def _fill(nnc, cache, lens, seed, dtype=F32):
    """Writes lens[b] rows to every sequence; returns them as the cache holds them, 64 bits, a list of [heads][n][d]."""
    g = _gen(seed)
    seq = _ints([b for b, n in enumerate(lens) for _ in range(n)])
    pos = _ints([i for n in lens for i in range(n)])
    k, v = (_randn(g, len(seq), cache.n_kv_heads, cache.head_dim, dtype=dtype) for _ in range(2))
    size = torch.exp2(torch.randint(-3, 3, (len(seq), 1, 1), generator=g, device="cuda").float()).to(dtype)
    v = v * size
    nnc.op_kv_write_paged(cache, k, v, pos, seq)
    held = (lambda x: quantise64(x)[0]) if cache.dtype is E4M3 else (lambda x: x.to(cache.dtype).double())
    return [[t.transpose(0, 1) for t in held(x).split(lens)] for x in (k, v)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=str)
@pytest.mark.parametrize("kv", [BF16, F16, E4M3], ids=str)
@pytest.mark.parametrize("page,heads,d", [(16, 1, 64), (64, 8, 128), (256, 3, 128), (32, 5, 64)])
def test_rows_come_back_as_the_cache_type_holds_them(nnc, dtype, kv, page, heads, d):
    lens = [0, 1, page - 1, page, page + 1, 3 * page + 5]
    cache = _paged(nnc, kv, lens, page, heads, d, 7)
    g = _gen(8)
    seq = _ints([b for b, n in enumerate(lens) for _ in range(n)])
    pos = _ints([i for n in lens for i in range(n)])
    k, v = (_randn(g, len(seq), heads, d, dtype=dtype) * torch.exp2(torch.randint(-12, 12, (len(seq), heads, 1), generator=g, device="cuda").to(dtype)) for _ in range(2))
    mix = torch.randperm(len(seq), generator=torch.Generator().manual_seed(1)).cuda()      # tokens in no order
    nnc.op_kv_write_paged(cache, k[mix].contiguous(), v[mix].contiguous(), pos[mix].contiguous(), seq[mix].contiguous())
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.to(kv).double())
    for out in (F32, BF16, F16):
        rk, rv = nnc.op_kv_read_paged(cache, pos, seq, dtype=out)
        assert rk.dtype is out
        assert torch.equal(rk, hold(k).to(out)) and torch.equal(rv, hold(v).to(out))
    if kv is E4M3:   # the codes and the exponents themselves
        where = cache.page_table[seq.long(), pos.long() // page].long(), pos.long() % page
        assert torch.equal(cache.k_scale[where[0], :, where[1]].double() - 127, quantise64(k)[1])
    # what no token named is what it was
    left = torch.ones(cache.k.shape[0], page, dtype=torch.bool, device="cuda")
    left[cache.page_table[seq.long(), pos.long() // page].long(), pos.long() % page] = False
    raw = cache.k.view(torch.uint8) if kv is E4M3 else cache.k
    old = raw.transpose(1, 2)[left]
    assert (old == 0x7f).all() if kv is E4M3 else old.isnan().all()
    assert nnc.op_status() == 0


def test_codes_of_rows_with_zeros_infinities_nan_and_extreme_sizes(nnc):
    cache = _paged(nnc, E4M3, [9], 16, 1, 64, 1)
    x = torch.zeros(9, 1, 64, device="cuda")
    x[1] = torch.linspace(-448, 448, 64, device="cuda")            # the largest code, scale 1
    x[2] = x[1] * 1.001                                            # just over: the next scale
    x[3, 0, :3] = torch.tensor([math.inf, -math.inf, 3.0])         # infinities saturate, the scale is the finite values'
    x[4, 0, :2] = torch.tensor([math.nan, 5.0])
    x[5] = 1e-30                                                   # below the smallest scale: 2^-60 stays, the value is 0
    x[6, 0, :2] = torch.tensor([3e38, 1.0])                        # above the largest: saturates
    x[7, 0, :4] = torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])   # the smallest code; halves go to even
    x[8] = 2.0 ** -130                                             # fp32 subnormals
    pos = _ints(range(9))
    nnc.op_kv_write_paged(cache, x, x, pos, _ints([0] * 9))
    k, v = nnc.op_kv_read_paged(cache, pos, _ints([0] * 9), dtype=F32)
    assert torch.equal(k.nan_to_num(nan=-1.25), v.nan_to_num(nan=-1.25))
    e = cache.k_scale[cache.page_table[0, 0].long(), 0, :9].int() - 127
    assert e.tolist() == [0, 0, 1, -7, -6, -60, 60, 0, -60]
    assert (k[0] == 0).all() and torch.equal(k[1].double(), quantise64(x[1])[0]) and torch.equal(k[2].double(), quantise64(x[2])[0])
    assert k[3, 0, :3].tolist() == [448 * 2.0 ** -7, -448 * 2.0 ** -7, 3.0]
    assert k[4, 0, 0].isnan() and k[4, 0, 1] == 5.0 and not k[4, 0, 1:].isnan().any()
    assert (k[5] == 0).all() and k[6, 0, 0] == 448 * 2.0 ** 60 and k[6, 0, 1] == 0
    assert k[7, 0, :4].tolist() == [448.0, 2.0 ** -9, 0.0, 2.0 ** -8]
    assert (k[8] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_rows_with_infinities_and_nan_anywhere(nnc, dtype, d):
    """Every row's scale is its own finite values', whatever its neighbours in the same warp hold."""
    g = _gen(d)
    x = _randn(g, 40, 3, d, dtype=dtype)
    for t in range(40):
        for h in range(3):
            kind = (3 * t + h) % 7
            at = (11 * t + 5 * h) % d
            if kind == 1: x[t, h, at] = math.inf
            if kind == 2: x[t, h, at] = -math.inf
            if kind == 3: x[t, h, at] = math.nan
            if kind == 4: x[t, h, at], x[t, h, (at + 9) % d] = math.nan, math.inf
            if kind == 5: x[t, h] = math.nan
            if kind == 6: x[t, h] = -math.inf
    y = x.flip(0).contiguous()
    cache = _paged(nnc, E4M3, [40], 16, 3, d, 1)
    pos, seq = _ints(range(40)), _ints([0] * 40)
    nnc.op_kv_write_paged(cache, x, y, pos, seq)
    for got, src, scale in zip(nnc.op_kv_read_paged(cache, pos, seq, dtype=F32), (x, y), (cache.k_scale, cache.v_scale)):
        finite = src.double().where(src.isfinite(), 0.0)
        want, e = quantise64(finite)
        assert torch.equal(got.isnan(), src.isnan())
        edge = 448 * power64(e)[..., None]
        want = torch.where(src == math.inf, edge, torch.where(src == -math.inf, -edge, want))
        assert torch.equal(got.double().where(~src.isnan(), 0.0), want.where(~src.isnan(), 0.0))
        at = cache.page_table[0, pos.long() // 16].long(), pos.long() % 16
        assert torch.equal(scale[at[0], :, at[1]].double() - 127, e)


def test_16_bit_rows_are_copied_bit_for_bit(nnc):
    for t in (BF16, F16):
        cache = _paged(nnc, t, [32], 16, 2, 64, 1)
        bits = torch.arange(32 * 2 * 64, device="cuda").mul(16).short().view(t).view(32, 2, 64)    # NaN and infinities among them
        pos, seq = _ints(range(32)), _ints([0] * 32)
        nnc.op_kv_write_paged(cache, bits, bits.flip(0).contiguous(), pos, seq)
        k, v = nnc.op_kv_read_paged(cache, pos, seq)
        assert torch.equal(k.view(torch.int16), bits.view(torch.int16)) and torch.equal(v.view(torch.int16), bits.flip(0).view(torch.int16))


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_padding_and_addresses_out_of_range_touch_nothing(nnc, kv):
    cache = _paged(nnc, kv, [40, 40], 16, 2, 64, 3)
    cache.page_table[1, 1] = 99        # no such page
    cache.page_table[1, 2] = -7
    _fill(nnc, cache, [16, 16], 9)
    assert nnc.op_status() == 0
    pools = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    same = lambda: all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in
                       zip(pools, [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]))
    x = torch.ones(3, 2, 64, device="cuda")
    out = [torch.full((3, 2, 64), 5.0, device="cuda") for _ in range(2)]
    # padding: a negative sequence or position is left out and is no error
    pos, seq = _ints([0, -1, -2 ** 31]), _ints([-1, 0, 1])
    nnc.op_kv_write_paged(cache, x, x, pos, seq)
    nnc.op_kv_read_paged(cache, pos, seq, out=out)
    assert same() and all((t == 5).all() for t in out) and nnc.op_status() == 0
    for p, s in ((48, 0), (2 ** 31 - 1, 0), (0, 2), (0, 2 ** 31 - 1), (16, 1), (32, 1)):
        pos, seq = _ints([p, -1, p]), _ints([s, 0, s])
        nnc.op_kv_write_paged(cache, x, x, pos, seq)
        torch.cuda.synchronize()
        with_status = nnc.op_status()
        assert same() and with_status == 0x100, (p, s)
        nnc.op_kv_read_paged(cache, pos, seq, out=out)
        torch.cuda.synchronize()
        assert all((t == 5).all() for t in out) and nnc.op_status() == 0x100, (p, s)
    assert nnc.op_status() == 0


def test_rows_from_fused_and_head_major_tensors_and_without_sequence_numbers(nnc):
    g = _gen(11)
    cache = _paged(nnc, BF16, [30, 30, 30], 16, 2, 128, 2)
    qkv = _randn(g, 3, 8, 128, dtype=BF16)
    pos = _ints([29, 0, 17])
    nnc.op_kv_write_paged(cache, qkv[:, 4:6], qkv[:, 6:8], pos)     # token t is sequence t's
    k, v = nnc.op_kv_read_paged(cache, pos)
    assert torch.equal(k, qkv[:, 4:6]) and torch.equal(v, qkv[:, 6:8])
    # into a contiguous [heads][max_seq][128] cache, rows 5 .. 7 of it
    flat = [torch.full((2, 20, 128), 3.0, dtype=BF16, device="cuda") for _ in range(2)]
    nnc.op_kv_read_paged(cache, pos, _ints([0, 1, 2]), out=[t.transpose(0, 1)[5:8] for t in flat])
    assert torch.equal(flat[0][:, 5:8].transpose(0, 1), qkv[:, 4:6]) and (flat[0][:, :5] == 3).all() and (flat[1][:, 8:] == 3).all()
    # and from one
    nnc.op_kv_write_paged(cache, flat[0].transpose(0, 1)[5:8], flat[1].transpose(0, 1)[5:8], _ints([1, 2, 3]), _ints([1, 1, 1]))
    k, _ = nnc.op_kv_read_paged(cache, _ints([3, 1, 3]), _ints([1, 1, 1]))       # the same row twice
    assert torch.equal(k, qkv[[2, 0, 2], 4:6])
    empty = torch.empty(0, 2, 128, dtype=BF16, device="cuda")
    nnc.op_kv_write_paged(cache, empty, empty, _ints([]), _ints([]))
    assert nnc.op_kv_read_paged(cache, _ints([]), _ints([]))[0].shape == (0, 2, 128)
    with pytest.raises(nnc.NncError):        # rows that are not 16-byte aligned
        odd = torch.zeros(3, 2, 129, dtype=BF16, device="cuda")[..., 1:]
        nnc.op_kv_write_paged(cache, odd, odd, pos)
    with pytest.raises(nnc.NncError):        # more tokens than sequences, without sequence numbers
        more = torch.zeros(4, 2, 128, dtype=BF16, device="cuda")
        nnc.op_kv_write_paged(cache, more, more, _ints([0, 1, 2, 3]))


# ---- attention ---------------------------------------------------------------------------------------------------------

def attend64(q, k, v, scale, window):
    """One sequence: q [heads][d], k, v [kv heads][n][d] in 64 bits; out, lse and what the bounds below are made of."""
    hq, d = q.shape
    h, n = k.shape[0], k.shape[1]
    first = max(0, n - window) if window else 0
    k, v = k[:, first:], v[:, first:]
    q = q.double().view(h, hq // h, d)
    s = torch.einsum("hgd,hnd->hgn", q, k) * scale
    reach = (torch.einsum("hgd,hnd->hgn", q.abs(), k.abs()) * abs(scale)).amax(-1)
    p = torch.softmax(s, -1)
    flat = lambda t: t.reshape(hq, *t.shape[2:])
    return flat(torch.einsum("hgn,hnd->hgd", p, v)), flat(torch.logsumexp(s, -1)), flat(torch.einsum("hgn,hnd->hgd", p, v.abs())), flat(reach)


def _check_attention(out, lse, q, held, lens, scale, window, kv):
    """fp32 part, with u = 2^-22 for a product-and-sum step of the tensor cores:
    scores: D / 16 steps of up to three terms each, the scalings (8 more), relative to sum |q k|; twice that in the weights
    (numerator and sum).  Weights: 2^-16 for two bf16 terms (16-bit results of a bf16 cache); for 16-bit results of codes one
    fp16 value (2^-11) with bf16 results and six more bits of a second one (2^-16) with fp16; within u otherwise.  Sums: a
    step per 16 positions of a warp's share, joins of warps and of CTAs, exp2 (32 more)."""
    k, v = held
    d = q.shape[-1]
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        want, want_lse, size, reach = attend64(q[b], k[b], v[b], scale, window)
        u = 2.0 ** -22
        score = u * (3 * d / 16 + 8) * reach
        sums = u * (n / 16 + 32)
        weights = {(BF16, BF16): 2.0 ** -16, (E4M3, BF16): 2.0 ** -11, (E4M3, F16): 2.0 ** -16}.get((kv, out.dtype), u)
        tol = torch.finfo(out.dtype).eps / 2 * want.abs() + (weights + sums + 2 * score)[..., None] * size
        tol += torch.finfo(F16).smallest_normal * 2.0 ** -11 if out.dtype is F16 else 0
        bad = (out[b].double() - want).abs() > tol
        assert not bad.any(), (b, n, bad.sum().item(), ((out[b].double() - want).abs() / tol).max().item())
        bad = (lse[b].double() - want_lse).abs() > score + sums + 2.0 ** -22 * want_lse.abs()
        assert not bad.any(), (b, n, (lse[b].double() - want_lse).abs().max().item())


TYPES = [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16), (BF16, F32), (F16, F32), (E4M3, F32)]


@pytest.mark.parametrize("kv,dtype", TYPES, ids=str)
@pytest.mark.parametrize("heads,group,d,page,window", [(1, 1, 128, 16, 0), (2, 4, 128, 64, 0), (8, 2, 64, 32, 0), (1, 8, 64, 256, 0), (2, 7, 128, 128, 100),
                                                       (1, 9, 64, 16, 0), (2, 16, 128, 64, 33), (1, 17, 128, 32, 0), (1, 40, 64, 64, 1), (3, 5, 64, 16, 250),
                                                       (2, 12, 64, 32, 0), (3, 32, 64, 256, 90), (2, 31, 128, 16, 0)])
def test_attention(nnc, scratch, kv, dtype, heads, group, d, page, window):
    lens = [0, 1, 15, 16, 17, 64, 0, 65, 127, 129, 700, 3]
    cache = _paged(nnc, kv, lens, page, heads, d, heads * 100 + group)
    held = _fill(nnc, cache, lens, group)
    if window:   # rows before the window must not be read either
        for b, n in enumerate(lens):
            for at in range(max(0, n - window)):
                pool = cache.k.view(torch.uint8) if kv is E4M3 else cache.k
                pool[cache.page_table[b, at // page].long(), :, at % page] = 0x7f if kv is E4M3 else math.nan
                pool = cache.v.view(torch.uint8) if kv is E4M3 else cache.v
                pool[cache.page_table[b, at // page].long(), :, at % page] = 0x7f if kv is E4M3 else math.nan
    q = _randn(_gen(d + group), len(lens), heads * group, d, dtype=dtype)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), window=window, scratch=scratch, want_lse=True)
    _check_attention(out, lse, q, held, lens, d ** -0.5, window, kv)
    assert nnc.op_status() == 0 and not scratch[:8192].any()
    again, lse2 = nnc.op_attn_decode_paged(q, cache, _ints(lens), window=window, scratch=scratch, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kv,dtype", [(BF16, BF16), (E4M3, F32), (F16, F16)], ids=str)
@pytest.mark.parametrize("batch,heads,group,length", [(1, 8, 4, 5000), (1, 1, 16, 30011), (300, 2, 2, 33), (37, 4, 3, 1024), (20, 1, 16, 2500), (8, 2, 32, 3001), (2, 1, 80, 9000)])
def test_attention_split_over_many_and_few_ctas(nnc, scratch, kv, dtype, batch, heads, group, length):
    lens = [length - (b * 37) % length for b in range(batch)]
    cache = _paged(nnc, kv, lens, 64, heads, 128, batch)
    held = _fill(nnc, cache, lens, batch + 1)
    q = _randn(_gen(batch), batch, heads * group, 128, dtype=dtype)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True, scale=0.2)
    _check_attention(out, lse, q, held, lens, 0.2, 0, kv)


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_attention_with_peaked_flat_and_extreme_scores(nnc, scratch, kv):
    lens = [513, 513, 513, 513, 513]
    cache = _paged(nnc, kv, lens, 16, 2, 64, 1)
    held = _fill(nnc, cache, lens, 2)
    q = _randn(_gen(3), 5, 8, 64)
    q[0] = 0                       # all scores alike
    q[1] *= 30                     # a few positions carry everything
    q[2] *= 1e-20
    q[3] *= 1e-38                  # subnormal products
    q[4, :, 0] = 1000.0            # one element above the others
    q = q.to(BF16)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    _check_attention(out, lse, q, held, lens, 64 ** -0.5, 0, kv)
    flat = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, scale=0.0, want_lse=True)
    _check_attention(*flat, q, held, lens, 0.0, 0, kv)


def test_attention_on_value_rows_of_very_different_scales(nnc, scratch):
    """Value rows from 2^-50 to 2^50: their scales ride on the exponents of the weights."""
    lens = [200]
    cache = _paged(nnc, E4M3, lens, 32, 1, 64, 1)
    g = _gen(1)
    pos, seq = _ints(range(200)), _ints([0] * 200)
    k, v = (_randn(g, 200, 1, 64) for _ in range(2))
    v *= torch.exp2(torch.randint(-50, 51, (200, 1, 1), generator=g, device="cuda").float())
    nnc.op_kv_write_paged(cache, k, v, pos, seq)
    held = [[quantise64(x)[0].transpose(0, 1)] for x in (k, v)]
    q = _randn(g, 1, 4, 64)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    _check_attention(out, lse, q, held, lens, 64 ** -0.5, 0, E4M3)


def test_attention_writes_its_rows_and_nothing_else(nnc, scratch):
    lens = [70, 0, 5, 16]
    cache = _paged(nnc, BF16, lens, 16, 2, 128, 6)
    held = _fill(nnc, cache, lens, 1)
    wide = _randn(_gen(2), 6, 3 * 4 * 128, dtype=BF16)               # rows of a wider matrix; two more rows than sequences
    q = wide[:3, 512:1024].unflatten(1, (4, 128))
    whole = torch.full((6, 1000), 9.0, dtype=BF16, device="cuda")
    out = whole[1:4, 8:520].unflatten(1, (4, 128))
    got, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens[:3]), scratch=scratch, out=out, want_lse=True)
    assert got.data_ptr() == out.data_ptr()
    _check_attention(out, lse, q, held, lens[:3], 128 ** -0.5, 0, BF16)
    whole[1:4, 8:520] = 9
    assert (whole == 9).all()
    assert nnc.op_attn_decode_paged(q[:0], cache, _ints([]), scratch=scratch).shape == (0, 4, 128)
    nan_q = q.clone()
    nan_q[0, 1] = math.nan                                            # a query's NaN is its own head's
    got = nnc.op_attn_decode_paged(nan_q, cache, _ints(lens[:3]), scratch=scratch)
    assert got[0, 1].isnan().all() and not got[0, [0, 2, 3]].isnan().any() and not got[1:].isnan().any()


def test_lengths_and_pages_out_of_range_are_cut_and_reported(nnc, scratch):
    lens = [48, 48]
    cache = _paged(nnc, BF16, lens, 16, 2, 64, 6)
    held = _fill(nnc, cache, lens, 1)
    q = _randn(_gen(2), 2, 4, 64, dtype=BF16)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints([49, -5]), scratch=scratch, want_lse=True)
    assert nnc.op_status() == 0x100
    _check_attention(out, lse, q, held, [48, 0], 0.125, 0, BF16)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints([2 ** 31 - 1, 48]), scratch=scratch, want_lse=True)
    assert nnc.op_status() == 0x100
    _check_attention(out, lse, q, held, [48, 48], 0.125, 0, BF16)
    for bad in (-1, 1 << 30):
        cache.page_table[0, 1] = bad                                  # positions 16 .. 31 are gone
        out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
        assert nnc.op_status() == 0x100
        keep = [i for i in range(48) if not 16 <= i < 32]
        gone = [[t[0][:, keep], t[1]] for t in held]
        _check_attention(out, lse, q, gone, [32, 48], 0.125, 0, BF16)
    cache.page_table[0] = -1                                          # none left: a row of zeros
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    assert nnc.op_status() == 0x100 and (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert nnc.op_status() == 0 and not scratch[:8192].any()


def test_attention_agrees_with_the_contiguous_cache_kernel(nnc, scratch):
    n = 777
    cache = _paged(nnc, BF16, [n, n], 64, 8, 128, 6)
    held = _fill(nnc, cache, [n, n], 1)
    kc, vc = (torch.stack(t).to(BF16).contiguous() for t in held)
    q = _randn(_gen(4), 2, 32, 128)
    # both keep fp32-level accuracy on two or three bf16 terms: 2^-16 of the weights, sums of 777 positions
    assert torch.allclose(nnc.op_attn_decode_paged(q, cache, _ints([n, n]), scratch=scratch), nnc.op_attn_decode(q, kc, vc, n), rtol=1e-4, atol=2e-5)


def test_pools_past_four_gigabytes(nnc, scratch):
    """Rows whose byte offset and whose element index pass 32 bits."""
    pages = 8400                                                      # 8 heads x 256 positions x 128: 512 KiB a page of bf16
    k = torch.empty(pages, 8, 256, 128, dtype=BF16, device="cuda")
    v = torch.empty(pages, 8, 256, 128, dtype=BF16, device="cuda")
    cache = nnc.PagedKV(k, v, _ints([[pages - 1, 0, pages - 2], [4097, 8191, 8192]]))
    lens = [600, 700]
    held = _fill(nnc, cache, lens, 1)
    q = _randn(_gen(4), 2, 32, 128, dtype=BF16)
    out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    _check_attention(out, lse, q, held, lens, 128 ** -0.5, 0, BF16)
    rk, _ = nnc.op_kv_read_paged(cache, _ints([0, 599]), _ints([0, 0]))
    assert torch.equal(rk.double(), held[0][0][:, [0, 599]].transpose(0, 1))


# ---- together ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_a_captured_decode_step_follows_its_sequences(nnc, scratch, kv):
    """Rotate, append, attend: captured once, replayed while positions and lengths move on in device memory; a second graph
    on a stream of its own with a scratch of its own runs beside it."""
    heads, group, d, page, steps = 2, 4, 128, 16, 40
    start = [0, 13, 30, 100]
    batch = len(start)
    freq, amp = nnc.rope_frequencies(d, 1e6, "ramp_index", 4.0, 64.0, 1.0, 8.0)
    g = _gen(17)
    stream_k, stream_v, stream_q = (_randn(g, batch, 200, n, d, dtype=BF16) for n in (heads, heads, heads * group))

    def lay(side):
        c = _paged(nnc, kv, [n + steps for n in start], page, heads, d, side)
        turned = []
        for b, n in enumerate(start):   # prompts
            p = torch.arange(n, device="cuda", dtype=torch.int32)
            nnc.op_kv_write_paged(c, nnc.op_rope(stream_k[b, :n], p, freq, amplitude=amp), stream_v[b, :n].contiguous(), p, torch.full_like(p, b))
            turned.append(nnc.op_rope(stream_k[b], torch.arange(200, device="cuda", dtype=torch.int32), freq, amplitude=amp))
        return c, turned

    def step_of(c, own_scratch):
        fused = torch.empty(batch, heads * (group + 2), d, dtype=BF16, device="cuda")
        pos, lens = _ints(start), _ints(start)
        out = torch.empty(batch, heads * group, d, dtype=BF16, device="cuda")
        nq = heads * group

        def run():
            lens.copy_(pos + 1)
            nnc.op_rope(fused[:, :nq + heads], pos, freq, amplitude=amp, out=fused[:, :nq + heads])
            nnc.op_kv_write_paged(c, fused[:, nq:nq + heads], fused[:, nq + heads:], pos)
            nnc.op_attn_decode_paged(fused[:, :nq], c, lens, scratch=own_scratch, out=out)
            pos.add_(1)
        return run, fused, pos, out

    graphs, sides = [], []
    for side in range(2):
        c, turned = lay(side)
        run, fused, pos, out = step_of(c, scratch if side == 0 else nnc.attn_paged_scratch())
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()                      # once outside the capture, then back
            pos.sub_(1)                # on the same stream
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
        graphs.append((graph, s, run))     # run holds the tensors that the graph works on
        sides.append((fused, pos, out, turned))
    hold = (lambda x: quantise64(x)[0]) if kv is E4M3 else (lambda x: x.double())
    for i in range(steps):
        at = [n + i for n in start]
        for (graph, s, _), (fused, pos, out, _) in zip(graphs, sides):
            with torch.cuda.stream(s):
                fused[:, :heads * group] = torch.stack([stream_q[b, at[b]] for b in range(batch)])
                fused[:, heads * group:heads * (group + 1)] = torch.stack([stream_k[b, at[b]] for b in range(batch)])
                fused[:, heads * (group + 1):] = torch.stack([stream_v[b, at[b]] for b in range(batch)])
                graph.replay()
        torch.cuda.synchronize()
        if i in (0, 1, 3, steps - 1):
            for fused, pos, out, turned in sides:
                assert pos.tolist() == [n + 1 for n in at]
                k = [hold(turned[b][:at[b] + 1]).transpose(0, 1) for b in range(batch)]
                v = [hold(stream_v[b, :at[b] + 1]).transpose(0, 1) for b in range(batch)]
                q = torch.stack([nnc.op_rope(stream_q[b, at[b]:at[b] + 1], _ints([at[b]]), freq, amplitude=amp)[0] for b in range(batch)])
                lse = torch.stack([attend64(q[b], k[b], v[b], d ** -0.5, 0)[1] for b in range(batch)])
                _check_attention(out, lse, q, (k, v), [n + 1 for n in at], d ** -0.5, 0, kv)
            assert torch.equal(sides[0][2], sides[1][2])
    assert nnc.op_status() == 0


def test_a_prefix_read_back_feeds_the_prompt_attention(nnc):
    """A paged prefix is read into a contiguous cache and nnc_op_attn_prefill continues it."""
    past, new, heads, group = 37, 20, 2, 2
    cache = _paged(nnc, E4M3, [past + new], 32, heads, 128, 6)
    held = _fill(nnc, cache, [past + new], 1)
    flat = [torch.zeros(1, heads, 64, 128, dtype=BF16, device="cuda") for _ in range(2)]
    pos = torch.arange(past + new, device="cuda", dtype=torch.int32)
    nnc.op_kv_read_paged(cache, pos, torch.zeros_like(pos), out=[t[0].transpose(0, 1)[:past + new] for t in flat])
    qkv = _randn(_gen(2), new, (heads * group + 2 * heads) * 128)
    hi, lo = nnc.op_attn_prefill(qkv, flat[0], flat[1], new, heads * group, past)
    got = (hi.double() + lo.double()).view(new, heads * group, 128)
    for t in range(new):
        want = attend64(qkv[t, :heads * group * 128].view(heads * group, 128), held[0][0][:, :past + t + 1], held[1][0][:, :past + t + 1], 128 ** -0.5, 0)
        # that kernel's weights and queries are two bf16 terms: 2^-16 of the scores' reach and of the sums, and its 2-term result
        assert ((got[t] - want[0]).abs() <= (2.0 ** -14 * (1 + want[3]))[:, None] * want[2]).all()


def test_other_streams_and_refusals_of_the_binding(nnc, scratch):
    lens = [300, 20]
    cache = _paged(nnc, BF16, lens, 64, 2, 128, 6)
    held = _fill(nnc, cache, lens, 1)
    q = _randn(_gen(2), 2, 8, 128, dtype=BF16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, lse = nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, want_lse=True)
    s.synchronize()
    _check_attention(out, lse, q, held, lens, 128 ** -0.5, 0, BF16)
    bad = [lambda: nnc.op_attn_decode_paged(q.float()[:, :, :64], cache, _ints(lens)),
           lambda: nnc.op_attn_decode_paged(q, cache, _ints(lens).long()),
           lambda: nnc.op_attn_decode_paged(q, cache, _ints(lens[:1])),
           lambda: nnc.op_attn_decode_paged(q, cache, torch.tensor(lens, dtype=torch.int32)),
           lambda: nnc.op_kv_write_paged(cache, q[:, :2], q[:, :2], _ints([0, 1]).long()),
           lambda: nnc.op_kv_write_paged(cache, q[:, :3], q[:, :3], _ints([0, 1])),
           lambda: nnc.op_kv_read_paged(cache, _ints([0]), _ints([0]), dtype=torch.float64),
           lambda: nnc.PagedKV(cache.k, cache.v[:1], cache.page_table),
           lambda: nnc.PagedKV(cache.k, cache.v, cache.page_table, torch.zeros(1, device="cuda"), None),
           lambda: nnc.op_rope(q, _ints([0, 1]), torch.zeros(64, device="cuda"))]
    bad += [lambda w=w: nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch, window=w) for w in (-1, 1 << 31, 1 << 32)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: nnc.op_attn_decode_paged(q.half(), cache, _ints(lens), scratch=scratch),
              lambda: nnc.op_attn_decode_paged(q[:, :7], cache, _ints(lens), scratch=scratch),
              lambda: nnc.op_attn_decode_paged(q, cache, _ints(lens), scratch=scratch[:1 << 20])):
        with pytest.raises(nnc.NncError):
            f()


def test_lists_past_their_count_are_refused_and_long_tables_are_not(nnc, scratch):
    """Tables that reach 2^30 positions: the list of tiles they allow is refused where it passes 2^30, and costs nothing else."""
    k, v = (torch.zeros(3, 1024, 16, 64, dtype=BF16, device="cuda") for _ in range(2))
    table = torch.full((2, 1 << 26), -1, dtype=torch.int32, device="cuda")
    table[0, :2] = _ints([2, 0])
    table[1, -1] = 1
    cache = nnc.PagedKV(k, v, table[:, :1 << 22].contiguous())
    with pytest.raises(nnc.NncError) as e:
        nnc.op_attn_decode_paged(torch.zeros(2, 1024, 64, dtype=BF16, device="cuda"), cache, _ints([1, 1]), scratch=scratch)
    assert e.value.status == -3
    few = nnc.PagedKV(k.view(3 * 1024, 1, 16, 64), v.view(3 * 1024, 1, 16, 64), table[:, :67000000].contiguous())
    x = _randn(_gen(1), 2, 1, 64, dtype=BF16)
    pos = 67000000 * 16 - 1
    few.page_table[1, -1] = 7
    nnc.op_kv_write_paged(few, x, x, _ints([17, pos]))
    nnc.op_kv_write_paged(few, x[:1], x[:1], _ints([16]), _ints([0]))
    out, lse = nnc.op_attn_decode_paged(x, few, _ints([18, pos + 1]), window=2, scratch=scratch, want_lse=True)
    assert nnc.op_status() == 0
    held = [[x[:1].double().transpose(0, 1).expand(1, 2, 64), torch.stack([torch.zeros(1, 64, device="cuda").double(), x[1].double()], 1)] for _ in range(2)]
    _check_attention(out, lse, x, held, [2, 2], 0.125, 0, BF16)


@pytest.mark.parametrize("kv", [BF16, E4M3], ids=str)
def test_calls_in_a_row_see_one_another(nnc, scratch, kv):
    """Rotate in place, append, attend, read back, over and over on the same buffers without a pause: every call works on what the one
    before it left, although their launches overlap."""
    heads, group, d, batch = 2, 2, 64, 300
    cache = _paged(nnc, kv, [200] * batch, 16, heads, d, 5)
    freq, _ = nnc.rope_frequencies(d)
    g = _gen(23)
    fused = _randn(g, batch, heads * (group + 2), d, dtype=BF16)
    start = fused.clone()
    nq, rounds = heads * group, 60
    seq = torch.arange(batch, device="cuda", dtype=torch.int32)
    pos = [torch.full((batch,), i, dtype=torch.int32, device="cuda") for i in range(rounds)]
    lens = [p + 1 for p in pos]
    outs, rows, turned = [], [], []
    for i in range(rounds):
        nnc.op_rope(fused[:, :nq + heads], pos[i], freq, out=fused[:, :nq + heads])        # turns the last round's result further
        nnc.op_kv_write_paged(cache, fused[:, nq:nq + heads], fused[:, nq + heads:], pos[i], seq)
        outs.append(nnc.op_attn_decode_paged(fused[:, :nq], cache, lens[i], scratch=scratch, want_lse=True))
        rows.append(nnc.op_kv_read_paged(cache, pos[i], seq, dtype=F32)[0])
        turned.append(fused[:, :nq + heads].clone())
    torch.cuda.synchronize()
    x = start.clone()
    hold = (lambda t: quantise64(t)[0]) if kv is E4M3 else (lambda t: t.double())
    keys = []
    for i in range(rounds):
        x[:, :nq + heads] = nnc.op_rope(x[:, :nq + heads], pos[i], freq)
        torch.cuda.synchronize()
        assert torch.equal(turned[i], x[:, :nq + heads])
        keys.append(hold(x[:, nq:nq + heads]))
        assert torch.equal(rows[i].double(), keys[-1])
    for i in (0, 1, 2, 17, 31, rounds - 1):
        k = torch.stack(keys[:i + 1], 2)                                                    # [batch][heads][positions][d]
        v = hold(start[:, nq + heads:])[:, :, None].expand(-1, -1, i + 1, -1)
        _check_attention(outs[i][0][:40], outs[i][1][:40], turned[i][:40, :nq], (k, v), [i + 1] * 40, d ** -0.5, 0, kv)
    assert nnc.op_status() == 0


def test_first_calls_may_be_captured(tmp_path):
    """A process whose first calls of the operations lie inside a stream capture."""
    import subprocess
    import sys
    prog = tmp_path / "child.py"
    prog.write_text("""
import sys, torch
sys.path[:0] = [%r, %r]
from paper_2512_21571_b200 import binding as nnc
cache = nnc.PagedKV.empty(4, 16, 1, 64, torch.bfloat16, 1, 2)
cache.page_table[0] = torch.arange(2)
x = torch.randn(1, 2, 64, device="cuda").to(torch.bfloat16)
pos, lens = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
freq, _ = nnc.rope_frequencies(64)
scratch = nnc.attn_paged_scratch()
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    y = nnc.op_rope(x, pos, freq)
    nnc.op_kv_write_paged(cache, y[:, :1], y[:, 1:], pos)
    out = nnc.op_attn_decode_paged(y, cache, lens, scratch=scratch)
    k, v = nnc.op_kv_read_paged(cache, pos)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(y, x) and torch.equal(k, x[:, :1]) and torch.equal(v, x[:, 1:])
assert torch.equal(out, x[:, 1:].expand(-1, 2, -1)) and nnc.op_status() == 0
print("captured")
""" % (__file__.rsplit("/tests/", 1)[0], __file__.rsplit("/tests/", 1)[0] + "/tests"))
    r = subprocess.run([sys.executable, str(prog)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
