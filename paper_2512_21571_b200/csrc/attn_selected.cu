// Attention of one new token per sequence over the pages that a list names for each of its KV heads.
//
// Positions are counted through the list (entry, then slot), so that a (sequence, KV head) is a run of tiles like any other; an entry's page
// is looked up one tile ahead of the copies.  Rows past the sequence's length (the last page's) are filled with zeros instead of read.
// Bound as the attention over all rows: by memory where there is enough of it (32 sequences, 64 pages of 64 for each of 8 heads: 94 us, 5.7 TB/s), by the
// beginning and the joining of few rows otherwise (20 sequences, 200 pages of 16 codes for each of 4 heads: 19 us, 29 MB).
#include "attn_paged_body.cuh"

namespace nnc {

namespace {

struct ListedRows {
    static constexpr bool kListed = true, kSums = false, kTypeF32 = true, kConcurrent = false;
    template <int TILE> static __device__ __forceinline__ Reach reach(const PagedAttnParams &p, int b, int head) {
        const int len = length_of(p, p.lens[b]);
        Reach r = reach_between<TILE>(0, len ? max(0, min(p.counts[(long long)b * p.c.n_kv + head], p.list_len)) << p.c.page_shift : 0);
        r.len = len;
        return r;
    }
    // page of the 16 positions from `pos` on, and how many of them the sequence has
    static __device__ __forceinline__ int page(const PagedAttnParams &p, const Place &at, int pos, int &rows) {
        rows = 0;
        const int entry = pos >> p.c.page_shift;
        if (!NNC_BC(entry < p.list_len && at.b < p.batch && at.head < p.c.n_kv, 3701)) return kNoPage;
        const int nth = p.list[((long long)at.b * p.c.n_kv + at.head) * p.list_len + entry];
        if ((unsigned)nth >= (unsigned)p.c.pages_per_seq) return kNoPage;
        rows = min(16, at.r.len - (nth << p.c.page_shift) - (pos & ((1 << p.c.page_shift) - 1)));
        if (rows <= 0) { rows = 0; return kNoRows; }
        return p.c.table[(long long)at.b * p.c.pages_per_seq + nth];
    }
    static long long most(const PagedAttnParams &p) { return (long long)p.list_len << p.c.page_shift; }
};

}  // namespace

cudaError_t launch_attn_selected(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, const int32_t *pages,
                                 const int32_t *counts, int list_len, void *out, float *lse, int type, int batch, int n_q_heads,
                                 int64_t q_stride, int64_t out_stride, float scale, void *scratch, size_t scratch_bytes) {
    PagedAttnParams p = paged_attn_params(lc, q, cache, lens, out, lse, batch, n_q_heads, q_stride, out_stride, scale, scratch, scratch_bytes);
    p.list = pages; p.counts = counts; p.list_len = list_len;
    return launch_paged_rows<ListedRows>(lc, p, cache, type);
}

}  // namespace nnc
