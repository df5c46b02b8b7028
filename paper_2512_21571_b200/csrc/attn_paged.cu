// Attention of one new token per sequence over everything (or the last `window` positions) that its sequence has in a paged cache.
#include "attn_paged_body.cuh"

namespace nnc {

namespace {

struct WholeRows {
    static constexpr bool kListed = false, kSums = false, kTypeF32 = true, kConcurrent = false;
    template <int TILE> static __device__ __forceinline__ Reach reach(const PagedAttnParams &p, int b, int) {
        const int len = length_of(p, p.lens[b]);
        return reach_between<TILE>((p.window > 0 && len > p.window) ? len - p.window : 0, len);
    }
    static __device__ __forceinline__ int page(const PagedAttnParams &p, const Place &at, int pos, int &) {
        if (!NNC_BC((pos >> p.c.page_shift) < p.c.pages_per_seq, 3207)) return kNoPage;
        return p.c.table[(long long)at.b * p.c.pages_per_seq + (pos >> p.c.page_shift)];
    }
    static long long most(const PagedAttnParams &p) { return (long long)p.c.pages_per_seq << p.c.page_shift; }   // positions a table allows
};

}  // namespace

cudaError_t launch_attn_paged(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, void *out, float *lse,
                              int type, int batch, int n_q_heads, int64_t q_stride, int64_t out_stride, float scale, int window,
                              void *scratch, size_t scratch_bytes) {
    PagedAttnParams p = paged_attn_params(lc, q, cache, lens, out, lse, batch, n_q_heads, q_stride, out_stride, scale, scratch, scratch_bytes);
    p.window = window;
    return launch_paged_rows<WholeRows>(lc, p, cache, type);
}

}  // namespace nnc
