"""Attention over the paged cache where its operands leave the ordinary: rows of zeros, scales at the ends of their range,
infinities, long shares.  Plain 64-bit forms and bounds as in test_gpu_paged."""

import pytest
import torch

from test_gpu_paged import BF16, E4M3, F32, _check_attention, _gen, _ints, _randn, nnc, quantise64, scratch  # noqa: F401

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
