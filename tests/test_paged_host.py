"""Host side of the paged-cache operations: what they refuse (before anything is launched; the pointers are never
followed, so this runs without a GPU) and the rotary frequencies against their definitions."""
import ctypes as C
import math

import pytest
import torch


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_b200 import build
    build.build()
    from paper_2512_21571_b200 import binding
    return binding


P = 4096   # a non-null, aligned address
INVALID, WORKSPACE, CAPACITY = -1, -2, -3


def _cache(nnc, **kw):
    f = dict(k=P, v=P, k_scale=None, v_scale=None, page_table=P, type=1, n_pages=9, page_size=64, n_kv_heads=2, head_dim=128,
             n_seqs=4, pages_per_seq=8)
    f.update(kw)
    return nnc.nnc_paged_kv(**f)


BAD_CACHES = [dict(k=None), dict(v=None), dict(page_table=None), dict(k=P + 8), dict(v=P + 2), dict(page_table=P + 2), dict(type=0),
              dict(type=4), dict(type=-1), dict(k_scale=P), dict(v_scale=P), dict(type=3), dict(type=3, k_scale=P),
              dict(type=3, k_scale=P, v_scale=P + 4), dict(n_pages=0), dict(n_pages=-1), dict(page_size=8), dict(page_size=48),
              dict(page_size=512), dict(page_size=0), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=256), dict(n_seqs=0),
              dict(pages_per_seq=0), dict(pages_per_seq=1 << 26)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_caches_that_are_refused(nnc, bad):
    ref = C.byref(_cache(nnc, **bad))
    assert nnc.lib.nnc_op_kv_write_paged(ref, P, P, 1, 1, 256, 128, P, P, None) == INVALID
    assert nnc.lib.nnc_op_kv_read_paged(ref, P, P, 1, 1, 256, 128, P, P, None) == INVALID
    assert nnc.lib.nnc_op_attn_decode_paged(P, ref, P, P, None, 0, 1, 4, 512, 512, 1.0, 0, P, 16 << 20, None) == INVALID


def test_row_calls_that_are_refused_and_empty_ones(nnc):
    c = _cache(nnc)
    ref = C.byref(c)
    good = dict(cache=ref, k=P, v=P, type=1, n=3, rs=256, hs=128, pos=P, seq=P)
    for fn in (nnc.lib.nnc_op_kv_write_paged, nnc.lib.nnc_op_kv_read_paged):
        call = lambda **kw: fn(*{**good, **kw}.values(), None)
        for bad in (dict(cache=None), dict(k=None), dict(v=None), dict(pos=None), dict(type=3), dict(type=-1), dict(n=-1), dict(k=P + 8),
                    dict(v=P + 4), dict(rs=252), dict(hs=4), dict(type=0, rs=130), dict(pos=P + 1), dict(seq=P + 2),
                    dict(seq=None, n=5)):
            assert call(**bad) == INVALID, bad
        assert call(n=0) == 0 and call(n=0, k=None, v=None, pos=None) == 0
    big = _cache(nnc, n_kv_heads=1 << 30)
    assert nnc.lib.nnc_op_kv_write_paged(C.byref(big), P, P, 1, 9, 256, 128, P, P, None) == CAPACITY


def test_attention_calls_that_are_refused_and_empty_ones(nnc):
    good = dict(q=P, cache=C.byref(_cache(nnc)), lens=P, out=P, lse=None, type=1, batch=4, nq=8, qs=1024, os=1024, scale=1.0, window=0,
                scratch=P, nbytes=16 << 20)
    call = lambda **kw: nnc.lib.nnc_op_attn_decode_paged(*{**good, **kw}.values(), None)
    codes = C.byref(_cache(nnc, type=3, k_scale=P, v_scale=P))
    half = C.byref(_cache(nnc, type=2))
    for bad in (dict(q=None), dict(cache=None), dict(lens=None), dict(out=None), dict(scratch=None), dict(type=2), dict(type=3), dict(type=-1),
                dict(cache=half, type=1), dict(cache=codes, type=3), dict(batch=-1), dict(batch=5), dict(nq=0), dict(nq=7), dict(nq=-8),
                dict(q=P + 8), dict(out=P + 8), dict(qs=1023), dict(os=4), dict(type=0, qs=1022), dict(window=-1), dict(lens=P + 2),
                dict(lse=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(nbytes=(16 << 20) - 1) == WORKSPACE and call(scratch=P + 128) == WORKSPACE and call(nbytes=0) == WORKSPACE
    assert call(batch=0) == 0 and call(batch=0, q=None, out=None, lens=None, scratch=None) == 0


def test_rope_calls_that_are_refused_and_empty_ones(nnc):
    good = dict(x=P, y=2 * P, type=1, n=3, heads=2, d=128, xr=256, xh=128, yr=256, yh=128, pos=P, freq=P, rot=128, inter=0, inv=0, amp=1.0)
    call = lambda **kw: nnc.lib.nnc_op_rope(*{**good, **kw}.values(), None)
    for bad in (dict(x=None), dict(y=None), dict(pos=None), dict(freq=None), dict(type=3), dict(type=-1), dict(n=-1), dict(heads=-1), dict(rot=0),
                dict(rot=-2), dict(rot=3), dict(rot=130), dict(d=2000, rot=64), dict(x=P + 1), dict(type=0, y=P + 2), dict(pos=P + 2), dict(freq=P + 4),
                dict(y=P, yr=512), dict(y=P, yh=64)):
        assert call(**bad) == INVALID, bad
    assert call(heads=1 << 24) == CAPACITY
    assert call(n=0) == 0 and call(heads=0) == 0 and call(n=0, x=None, y=None, pos=None, freq=None) == 0


def test_frequencies_follow_their_definitions(nnc):
    d, theta, factor, original = 48, 5e5, 8.0, 4096.0
    f0 = [theta ** (-2 * i / d) for i in range(d // 2)]
    get = lambda *a, **kw: nnc.rope_frequencies(*a, device="cpu", **kw)
    close = lambda got, want: torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-14, atol=0)
    f, amp = get(d, theta)
    assert f.dtype == torch.float64 and close(f, f0) and amp == 1.0
    f, amp = get(d, theta, "linear", factor)
    assert close(f, [x / factor for x in f0]) and amp == 1.0
    f, amp = get(d, theta, "base", factor)
    assert close(f, [(theta * factor ** (d / (d - 2))) ** (-2 * i / d) for i in range(d // 2)])
    assert math.isclose(f[-1], f0[-1] / factor, rel_tol=1e-13) and f[0] == 1.0
    f, amp = get(d, theta, "ramp_turns", factor, original, 1.0, 4.0)
    want = []
    for x in f0:
        turns = original * x / (2 * math.pi)
        g = min(1.0, max(0.0, (turns - 1.0) / 3.0))
        want.append(x * (g + (1 - g) / factor))
    assert close(f, want) and amp == 1.0
    assert f[0] == 1.0 and math.isclose(f[-1], f0[-1] / factor, rel_tol=1e-14)
    f, amp = get(d, theta, "ramp_index", factor, original, 1.0, 32.0)
    at = lambda turns: d * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
    lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), d - 1)
    want = []
    for i, x in enumerate(f0):
        g = 1 - min(1.0, max(0.0, (i - lo) / (hi - lo)))
        want.append(x * (g + (1 - g) / factor))
    assert close(f, want) and math.isclose(amp, 0.1 * math.log(factor) + 1, rel_tol=1e-6)
    f, amp = get(d, theta, "ramp_index", 1.0, original, 1.0, 32.0)
    assert close(f, f0) and amp == 1.0
    f, _ = get(2, theta, "ramp_index", factor, original, 1.0, 32.0)     # one pair
    assert f.numel() == 1 and 1 / factor <= f.item() <= 1.0


def test_frequencies_that_are_refused(nnc):
    out = (C.c_double * 64)()
    call = lambda *a: nnc.lib.nnc_rope_frequencies(*a, out, None)
    assert call(64, 1e6, 0, 0.0, 0.0, 0.0, 0.0) == 0
    nan = math.nan
    for bad in ((0, 1e6, 0, 1., 1., 1., 2.), (63, 1e6, 0, 1., 1., 1., 2.), (-2, 1e6, 0, 1., 1., 1., 2.), (64, 0., 0, 1., 1., 1., 2.),
                (64, nan, 0, 1., 1., 1., 2.), (64, 1e6, 5, 2., 1., 1., 2.), (64, 1e6, -1, 2., 1., 1., 2.), (64, 1e6, 1, .5, 1., 1., 2.),
                (64, 1e6, 1, nan, 1., 1., 2.), (2, 1e6, 2, 2., 1., 1., 2.), (64, 1e6, 3, 2., 0., 1., 2.), (64, 1e6, 3, 2., 1., 0., 2.),
                (64, 1e6, 3, 2., 1., 2., 2.), (64, 1e6, 4, 2., nan, 1., 2.), (64, 1., 4, 2., 1., 1., 2.)):
        assert call(*bad) == INVALID, bad
    assert nnc.lib.nnc_rope_frequencies(64, 1e6, 0, 1., 1., 1., 2., None, None) == INVALID
    with pytest.raises(ValueError):
        nnc.rope_frequencies(64, scaling="cubic", device="cpu")


def test_tensors_on_the_host_are_refused(nnc):
    x = torch.zeros(2, 2, 64)
    with pytest.raises(ValueError):
        nnc.op_rope(x, torch.zeros(2, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        nnc.PagedKV(torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16),
                    torch.zeros(1, 1, dtype=torch.int32))
