// What the kernels of the attention behind a shared prefix have in common: groups of sequences, the list of tiles, scratch.
#pragma once
#include "paged.cuh"

namespace nnc {

constexpr int kPrefixRows = 128;       // query rows of a tile, at most: as many sequences' as fit, all query heads of the KV head each
constexpr int kPrefixStep = 64;        // positions of a step
constexpr int kPrefixFixed = 2;        // places in the list for what it costs to begin and to end a tile, in steps
constexpr int kPrefixMaxCtas = 160;    // one per SM

struct PrefixGroups {
    const int32_t *starts, *shared;
    int n_groups, batch;
    int least;                         // sequences that a group has at least where its rows are read for all of them at once
};

// a group's tiles
struct PrefixPlan {
    long long base;                    // first place in the list, where it is known
    int b0, members, tiles, steps;     // first sequence, sequences, tiles per KV head, steps of a tile (0: no prefix)
    int prefix;                        // positions
};
// what the joining kernel wants to know of a sequence
struct PrefixOf {
    long long first, row;              // first place of its tile of KV head 0, first row of its queries for KV head 0 (of CTA 0)
    long long per_head;                // places from one KV head to the next
    int rows_per_head, steps;          // steps 0: nothing from a prefix
    long long share;                   // places of a CTA
};

__device__ __forceinline__ int first_of(const PrefixGroups &s, int g) { return min(max(s.starts[g], 0), s.batch); }
__device__ __forceinline__ int members_of(const PrefixGroups &s, int g) { return max(first_of(s, g + 1) - first_of(s, g), 0); }

// positions of a group that its sequences share: whole pages; none where there are too few sequences for it to pay
__device__ __forceinline__ int prefix_of(const PagedView &c, const PrefixGroups &s, int g) {
    if (members_of(s, g) < s.least) return 0;
    return min(max(s.shared[g], 0), c.pages_per_seq << c.page_shift) >> c.page_shift << c.page_shift;
}

// A sequence that ends inside its group's prefix reads its own rows alone: so every query that meets the shared rows attends to all of
// them, and nothing behind a sequence's end is multiplied by its weights of 0 (which makes NaN of infinities).
__device__ __forceinline__ bool takes_prefix(int prefix, int len) { return len >= prefix; }

// the group of a sequence, or -1 (whatever `starts` holds, the answer lies in range)
__device__ __forceinline__ int group_of(const PrefixGroups &s, int b) {
    int lo = -1, hi = s.n_groups;      // starts[lo] <= b < starts[hi], where these exist
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.starts[mid] <= b) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && b < s.starts[lo + 1] ? lo : -1;
}

__device__ __forceinline__ PrefixPlan plan_of(const PagedView &c, const PrefixGroups &s, int g, int per_tile) {   // per_tile: sequences
    PrefixPlan p;
    p.b0 = first_of(s, g);
    p.members = members_of(s, g);
    p.tiles = (p.members + per_tile - 1) / per_tile;
    p.prefix = prefix_of(c, s, g);
    p.steps = p.members ? (p.prefix + kPrefixStep - 1) / kPrefixStep : 0;
    p.base = 0;
    return p;
}
__device__ __forceinline__ long long places_of(const PagedView &c, const PrefixPlan &p) {
    return p.steps ? (long long)c.n_kv * p.tiles * (p.steps + kPrefixFixed) : 0;
}

// Partial results: a row for every query row of a (tile, CTA) pair that occurs.  Pairs in the list's order move on by a tile's rows or by
// a CTA, so row (rows of earlier tiles) + 128 CTA is a pair's own.
struct PrefixScratch {
    PrefixPlan *plan;                  // [n_groups]: what the CTA that writes `of` makes it from
    PrefixOf *of;                      // [batch]: for the joining kernel
    float2 *ml;                        // [rows]: reference in log2 units, sum
    float4 *o;                         // [D / 4][rows]: neighbouring threads hold neighbouring rows
    float2 *tail_ml;                   // [batch][n_q]
    float *tail;                       // [batch][n_q][D]: what lies behind the prefix, the same way
};

// whether that kernel takes sequences of such a cache: asked before anything is launched
bool attn_tail_fits(const nnc_paged_kv &cache, int batch);
cudaError_t launch_attn_tail(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, const PrefixGroups &groups, float *out,
                             float2 *ml, int type, int n_q_heads, int64_t q_stride, float scale, void *scratch, size_t scratch_bytes);

}  // namespace nnc
