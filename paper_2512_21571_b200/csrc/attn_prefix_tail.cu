// Attention of one new token per sequence over what lies behind the positions that its group shares, as sums in 32 bits with their weights: one part
// of the attention behind a shared prefix.  26 us for 80 MB behind 64 sequences' prefix, some of them while the prefix's last CTAs run.
#include "attn_paged_body.cuh"
#include "attn_prefix.cuh"

namespace nnc {

namespace {

struct TailRows {
    static constexpr bool kListed = false, kSums = true, kTypeF32 = false, kConcurrent = true;
    template <int TILE> static __device__ __forceinline__ Reach reach(const PagedAttnParams &p, int b, int) {
        const PrefixGroups groups{p.starts, p.shared, p.n_groups, p.batch, p.least};
        const int len = length_of(p, p.lens[b]), g = group_of(groups, b);
        const int prefix = g < 0 ? 0 : prefix_of(p.c, groups, g), start = takes_prefix(prefix, p.lens[b]) ? prefix : 0;
        return start < len ? reach_between<TILE>(start, len) : Reach{len, len, 0, len};
    }
    static __device__ __forceinline__ int page(const PagedAttnParams &p, const Place &at, int pos, int &) {
        if (!NNC_BC((pos >> p.c.page_shift) < p.c.pages_per_seq, 3501)) return kNoPage;
        return p.c.table[(long long)at.b * p.c.pages_per_seq + (pos >> p.c.page_shift)];
    }
    static long long most(const PagedAttnParams &p) { return (long long)p.c.pages_per_seq << p.c.page_shift; }
};

}  // namespace

bool attn_tail_fits(const nnc_paged_kv &c, int batch) {
    const int tile = c.head_dim == 64 ? (c.type == NNC_E4M3 ? Shape<64, 1, NNC_E4M3, NNC_BF16>::kTile : Shape<64, 1, NNC_BF16, NNC_BF16>::kTile)
                                      : (c.type == NNC_E4M3 ? Shape<128, 1, NNC_E4M3, NNC_BF16>::kTile : Shape<128, 1, NNC_BF16, NNC_BF16>::kTile);
    return list_fits((long long)c.pages_per_seq * c.page_size, tile, batch, c.n_kv_heads);
}

cudaError_t launch_attn_tail(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, const PrefixGroups &groups, float *out,
                             float2 *ml, int type, int n_q_heads, int64_t q_stride, float scale, void *scratch, size_t scratch_bytes) {
    PagedAttnParams p = paged_attn_params(lc, q, cache, lens, out, (float *)ml, groups.batch, n_q_heads, q_stride, (int64_t)n_q_heads * cache.head_dim, scale, scratch,
                                          scratch_bytes);
    p.starts = groups.starts; p.shared = groups.shared; p.n_groups = groups.n_groups; p.least = groups.least;
    return launch_paged_rows<TailRows>(lc, p, cache, type);
}

}  // namespace nnc
