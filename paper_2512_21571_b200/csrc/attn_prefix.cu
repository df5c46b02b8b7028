// Attention of one new token per sequence where groups of sequences share the first positions of a paged cache: the shared rows are read
// once for the whole group.
//
//   s_n = scale q.k_n,  o = sum_n exp(s_n - m) v_n / sum_n exp(s_n - m),  n < lens[b], in three launches:
//   prefix   (this file)  m, l = sum exp(s_n - m), o~ = sum exp(s_n - m) v_n over the shared positions, for all queries of a group at a time
//   tail     (attn_prefix_tail.cu)  the same over what lies behind them, sequence by sequence
//   joining  (this file)  both; m and l go from one to the other as they are, so that a weight is as exact between parts as within one
//
// The queries of a group's sequences for one KV head are rows of one operand, so the prefix is a pair of matrix products with up to 128
// rows, and tcgen05 does them: S = Q K^T and O += P V with S, P and O in tensor memory, K and V pages fetched by TMA (a page of a KV head is a
// [page_size][head_dim] matrix; boxes of 16 to 64 positions, zeros where a page is missing).  Bound by the softmax's
// steps: some 0.5 us each (64 positions of 128 rows), of which the tensor cores need 0.2 to 0.4 and the exponentials 0.27; its warps wait for their
// scores, tensor memory and each other, and issue in 0.4 of a scheduler's slots.  25 us for 64 sequences of 32 heads behind 8192 positions
// (34 MB; 1.3 TB/s).
//   - The list of (group, KV head, tile, step of 64 positions) is cut into one contiguous share per CTA; the groups' lengths live on the
//     device, so every CTA adds up the list itself.  A share may begin and end inside a tile.
//   - One CTA per SM: a warp that fetches K (and Q), one that fetches V, one that issues S = Q K^T, one that issues O += P V (a single warp's
//     instructions for two of these take longer than the step), and two teams of four softmax warps with a query row per thread, which take
//     turns at the steps (three teams for heads of 64, whose accumulators leave room for a third: 48 sequences of 24 such heads behind 65536
//     positions 65 us instead of 70).  Four score buffers in tensor memory, so that scores run two steps ahead (with two, a step's scores wait for the
//     product of the step before it).  Each team has an output accumulator and a running maximum of its own; they are joined where a share's
//     part of a tile ends.
//   - E4M3: codes times their rows' scales are bf16 values exactly (down to 2^-133).  They come to shared memory as they are, eight warps make
//     the rows of them that the products read, half of them a step each, and the two teams hold half of a step's scores at a time, which leaves
//     room for the registers of 640 threads.  (Five groups of 12 behind up to 6000 codes: 65 us; all eight warps at every step, with one team or
//     two, 70; four and one team 73, four and two 75; every sequence's rows by themselves 112.)
//   - Queries enter exactly.  Probabilities are two terms of the cache's type (bf16: 16 bits, fp16: 22), written over the scores they
//     come from: one bf16 term alone would add an error of the size of the result's own rounding.  fp32 queries and results would need three
//     terms and shorter sums; they go through the kernel that reads every sequence's rows.
#include <cuda_fp16.h>

#include <type_traits>

#include "attn_prefill_common.cuh"
#include "attn_prefix.cuh"

namespace nnc {

namespace {

constexpr int kSoftmaxRows = 128;
constexpr int kScoreBuffers = 4;
constexpr uint32_t kColS = 0, kColO = kScoreBuffers * kPrefixStep, kTmemColumns = 512;   // score buffers, then the teams' accumulators
// The reference of sums whose weights are all 0, where they are infinities or NaN all the same (of values); of sums of nothing it is -infinity
constexpr float kNothing = -3e38f;
constexpr float kLn2 = 0.69314718055994530942f;

template <int D, bool CODES> struct Tiles {
    static constexpr int kTeams = D == 64 && !CODES ? 3 : 2;     // of four softmax warps; tensor memory has an accumulator for each
    static constexpr int kThreads = 128 + 128 * kTeams + (CODES ? 256 : 0);
    static constexpr int kHalves = D / 64;                        // slabs of 64 elements
    static constexpr int kQSlab = kPrefixRows * 128, kQ = kHalves * kQSlab;
    static constexpr int kSlabKV = kPrefixStep * 128, kKV = kHalves * kSlabKV;
    // of K and of V.  At most kScoreBuffers: who fills a stage takes it as free by the barriers of its step's score buffer, which then cannot move on by
    // more than one phase before it has looked
    static constexpr int kStages = 4 - (CODES && D == 128);
    static_assert(kStages <= kScoreBuffers, "");
    // codes as they come: K, V, then a scale byte a row of each
    static constexpr int kCodes = kPrefixStep * D, kRaw = 2 * kCodes + 2 * kPrefixStep, kRawStages = CODES ? 4 : 0, kRawAt = kQ + 2 * kStages * kKV;
    static constexpr int kBars = kRawAt + kRawStages * kRaw;
    // more than an SM has left beside it for a CTA of the tail, which would take turns with the softmax (171 us instead of 89 + 14)
    static constexpr int kSmem = (kBars > 160 << 10 ? kBars : 160 << 10) + 1024 /*alignment*/ + 512 /*barriers*/;
};

struct PrefixParams {
    PagedView c;
    PrefixGroups groups;
    PrefixScratch s;
    const int32_t *lens;
    long long part_rows;
    int group, per_tile, n_q, box;      // query heads per KV head; sequences of a tile; query heads in all; positions of a TMA box
    uint32_t flip;                      // the sign bit of the scores where the scale is negative
    float scale_log2;                   // |scale| in log2 units
    int *wait_status;
};

// a step, and its place in the list
struct Step {
    PrefixPlan plan;
    long long index;
    int g, head, tile, step;
};

// the first group from g on that has a prefix
__device__ __forceinline__ void find_group(const PrefixParams &p, Step &at) {
    for (at.plan.steps = 0; at.g < p.groups.n_groups; ++at.g) {
        at.plan = plan_of(p.c, p.groups, at.g, p.per_tile);
        if (at.plan.steps) return;
    }
}
__device__ __forceinline__ void advance(const PrefixParams &p, Step &at) {
    ++at.index;
    if (++at.step < at.plan.steps) return;
    at.index += kPrefixFixed;
    at.step = 0;
    if (++at.tile < at.plan.tiles) return;
    at.tile = 0;
    if (++at.head < p.c.n_kv) return;
    at.head = 0;
    ++at.g;
    find_group(p, at);
}

__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}

// two floats to nearest even, the first in the low half: one instruction
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void store16(float4 *dst, const uint32_t *v) {
    *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ float top3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The products are issued by warp-wide code in which one lane's instruction counts: what they address then lies in uniform registers.  (Inside a
// branch that one lane takes, every operand is moved there first: 85 to 115 cycles an instruction instead of 50.)
__device__ __forceinline__ void mma_ss(bool one, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)one) : "memory");
}
__device__ __forceinline__ void mma_ts(bool one, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {   // the first operand in tensor memory
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)one) : "memory");
}
__device__ __forceinline__ void mma_commit(bool one, uint32_t bar) {
    asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"((uint32_t)one) : "memory");
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_more(uint32_t bar, uint32_t bytes) {   // without arriving
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// KV: the cache's type; queries are of that type, or bf16 for codes
template <int D, int KV>
__global__ void __launch_bounds__(Tiles<D, KV == NNC_E4M3>::kThreads, 1)
attn_prefix_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const PrefixParams p) {
    constexpr bool CODES = KV == NNC_E4M3, BF = KV != NNC_F16;
    typedef Tiles<D, CODES> T;
    constexpr int kThreads = T::kThreads, kTeams = T::kTeams;
    constexpr int kHeld = CODES ? 1 : 2;           // halves of a step's scores that a thread holds at a time
    constexpr int NS = T::kStages, NC = T::kRawStages;
    // fp16 probabilities are scaled by 2^6, so that small ones keep their bits (at most 2^8 by the lazy maximum: below 2^15; sums are scaled alike)
    constexpr float kLift = BF ? 0.f : 6.f;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_tile = base;
    auto k_tile = [&](int st) { return base + (uint32_t)(T::kQ + st * 2 * T::kKV); };
    auto v_tile = [&](int st) { return k_tile(st) + (uint32_t)T::kKV; };
    const uint32_t q_ready = base + (uint32_t)T::kBars;
    auto k_full = [&](int st) { return q_ready + 8u * (1 + st); };
    auto v_full = [&](int st) { return q_ready + 8u * (1 + NS + st); };
    auto s_full = [&](int j) { return q_ready + 8u * (1 + 2 * NS + j % kScoreBuffers); };                           // by step
    auto p_full = [&](int j) { return q_ready + 8u * (1 + 2 * NS + kScoreBuffers + j % kScoreBuffers); };
    auto pv_done = [&](int j) { return q_ready + 8u * (1 + 2 * NS + 2 * kScoreBuffers + j % kScoreBuffers); };
    auto turn = [&](int j) { return (uint32_t)(j / kScoreBuffers & 1); };                                            // their parity
    auto raw_full = [&](bool v, int st) { return q_ready + 8u * (1 + 2 * NS + 3 * kScoreBuffers + (v ? NC : 0) + st); };   // codes
    auto raw_free = [&](bool v, int st) { return q_ready + 8u * (1 + 2 * NS + 3 * kScoreBuffers + 2 * NC + (v ? NC : 0) + st); };
    auto raw_tile = [&](bool v, int st) { return base + (uint32_t)(T::kRawAt + st * T::kRaw + (v ? T::kCodes : 0)); };
    auto raw_scales = [&](bool v, int st) { return base + (uint32_t)(T::kRawAt + st * T::kRaw + 2 * T::kCodes + (v ? kPrefixStep : 0)); };
    constexpr int kConverters = 64, kFillers = CODES ? kConverters : 1;   // arrivals that make a stage full: two warps, or the copy's
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s, first_g;
    __shared__ long long first_rest, sums[kThreads / 32];
    __shared__ float2 ml_s[kTeams][kPrefixRows];
    __shared__ uint32_t odd_s[CODES ? 1 : D];   // what a part's values hold besides finite numbers, where somebody looked: infinity 1, -infinity 2, NaN 4
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // the same in all lanes, which the compiler then knows
    volatile int *abort_flag = &abort_s;
    if (tid == 0) {
        abort_s = 0;
        mbar_init(q_ready, 1);
        for (int st = 0; st < NS; ++st) { mbar_init(k_full(st), kFillers); mbar_init(v_full(st), kFillers); }
        for (int st = 0; st < NC; ++st)
            for (int v = 0; v < 2; ++v) { mbar_init(raw_full(v, st), 1); mbar_init(raw_free(v, st), kConverters); }
        for (int j = 0; j < kScoreBuffers; ++j) { mbar_init(s_full(j), 1); mbar_init(p_full(j), kSoftmaxRows); mbar_init(pv_done(j), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();   // groups, lengths, tables, queries and rows may be the preceding kernel's
    pdl_launch_dependents();   // after that: the tail does not wait for this kernel, and what came before is done for it too
    // ---- the list: its length, and where this CTA's share begins ----
    const int per = (p.groups.n_groups + kThreads - 1) / kThreads, g_lo = min(tid * per, p.groups.n_groups), g_hi = min(g_lo + per, p.groups.n_groups);
    long long mine = 0;
    for (int g = g_lo; g < g_hi; ++g) mine += places_of(p.c, plan_of(p.c, p.groups, g, p.per_tile));
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sums[warp] = incl;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) { if (w < warp) before += sums[w]; total += sums[w]; }
    before += incl - mine;
    const long long share = max((total + gridDim.x - 1) / gridDim.x, 1ll), cta = blockIdx.x;
    const long long t0 = cta * share, t1 = min(t0 + share, total);
    if (cta == gridDim.x - 1) {   // this CTA, whose share is the shortest, writes what the joining kernel wants to know (below); and looks the groups over
        long long at = before;
        for (int g = g_lo; g < g_hi; ++g) {
            PrefixPlan plan = plan_of(p.c, p.groups, g, p.per_tile);
            plan.base = at;
            at += places_of(p.c, plan);
            p.s.plan[g] = plan;
            const bool orderly = p.groups.starts[g] >= 0 && p.groups.starts[g] <= p.groups.starts[g + 1] && p.groups.starts[g + 1] <= p.groups.batch;
            if (!orderly || p.groups.shared[g] < 0 || p.groups.shared[g] > (p.c.pages_per_seq << p.c.page_shift)) paged_complain(p.c);
        }
    }
    if (t0 < t1 && t0 >= before && t0 - before < mine) {
        long long rest = t0 - before;
        int g = g_lo;
        for (; g < g_hi; ++g) {
            const long long n = places_of(p.c, plan_of(p.c, p.groups, g, p.per_tile));
            if (rest < n) break;
            rest -= n;
        }
        first_g = g;
        first_rest = rest;
    }
    __syncthreads();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    if (cta == gridDim.x - 1)
        for (int b = tid; b < p.groups.batch; b += kThreads) {
            PrefixOf of = {};
            const int g = group_of(p.groups, b);
            if (g >= 0) {
                const PrefixPlan plan = p.s.plan[g];
                const int nth = b - plan.b0;
                of.per_head = (long long)plan.tiles * (plan.steps + kPrefixFixed);
                of.first = plan.base + (long long)(nth / p.per_tile) * (plan.steps + kPrefixFixed);
                of.rows_per_head = plan.members * p.group;
                of.row = (long long)plan.b0 * p.n_q + (long long)nth * p.group;
                of.steps = takes_prefix(plan.prefix, p.lens[b]) ? plan.steps : 0;
                of.share = share;
            }
            p.s.of[b] = of;
        }
    Step at = {};
    at.index = t1;
    if (t0 < t1) {
        at.g = first_g;
        at.plan = plan_of(p.c, p.groups, at.g, p.per_tile);
        const int per_tile = at.plan.steps + kPrefixFixed;
        const long long item = first_rest / per_tile;
        at.step = (int)(first_rest - item * per_tile);
        at.head = (int)(item / at.plan.tiles);
        at.tile = (int)(item - (long long)at.head * at.plan.tiles);
        at.index = t0;
        if (at.step >= at.plan.steps) {   // a place after a tile's steps: on to the next tile
            at.index += at.plan.steps - 1 - at.step;
            at.step = at.plan.steps - 1;
            advance(p, at);
        }
    }

    long long all = 0;   // steps of this share
    for (Step s = at; s.index < t1 && s.g < p.groups.n_groups;) {   // a tile's at a time
        const long long n = min((long long)(s.plan.steps - s.step), t1 - s.index);
        all += n;
        s.index += n - 1;
        s.step += (int)n - 1;
        advance(p, s);
    }
    const int steps = __shfl_sync(0xffffffffu, (int)min(all, 0x7fffffffll), 0);

    // how many steps this share has of the tile where `x` stands, which then moves to the next tile
    auto part = [&](Step &x) -> int {
        const int n = __shfl_sync(0xffffffffu, (int)min((long long)(x.plan.steps - x.step), t1 - x.index), 0);
        x.index += n - 1;
        x.step += n - 1;
        advance(p, x);
        return n;
    };
    auto wait = [&](uint32_t bar, uint32_t parity, int code) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.wait_status, code)); };

    // Queries: a tile's first when the share begins, another's when the last scores of the tile before it are complete.  Rows of 16 bits: the warp that
    // fetches K waits for that and goes on looking until there is no tile left.  Codes: that warp waits for conversions, which say too little of the
    // scores (a barrier tells its last two phases apart), so the warp that issues the scores asks for the queries.
    Step tile_q = at;
    int begins_q = 0;   // the step where the next tile to load the queries of begins
    auto load_queries = [&]() {   // [sequence][query head of the KV head][64]: a row of the tile after the other
        if (lane == 0) mbar_expect_tx(q_ready, (uint32_t)(T::kHalves * p.per_tile * p.group * 128));
        __syncwarp();
        if (lane < T::kHalves) tma_load_3d(q_tile + lane * T::kQSlab, &map_q, q_ready, 64 * lane, tile_q.head * p.group, tile_q.plan.b0 + tile_q.tile * p.per_tile);
        begins_q += part(tile_q);
    };
    // stage of step j (K's or V's) is free when the product that reads it is complete: the scores of step j - NS, or the output's
    auto wait_stage = [&](bool v, int j) -> bool { return wait(v ? pv_done(j - NS) : s_full(j - NS), turn(j - NS), v ? 42 : 41); };

    if (warp <= 1) {   // ---------------- TMA producers, a lane a box: keys and queries; values ----------------
        const bool v = warp == 1;
        // this lane's half of the head's elements, first position of a step; of codes: the box, or its scales
        const int half = lane & 1, r = (lane >> 1) * p.box;
        const bool loads = (CODES || half < T::kHalves) && r < kPrefixStep;
        const CUtensorMap *const map = v ? &map_v : &map_k;
        const int absent = (int)min(paged_rows(p.c), 0x7fffffffll);   // a row outside the tensor: zeros
        const int page_rows = p.c.n_kv << p.c.page_shift, page_mask = (1 << p.c.page_shift) - 1;
        if (!CODES && steps > 0 && !v) load_queries();
        int left = 0, pos = 0, head_rows = 0, end = 0, page = 0;
        const int32_t *table = p.c.table;
        for (int j = 0, st = 0, turn_st = 1; j < steps || (!CODES && !v && begins_q < steps); ++j) {
            if constexpr (CODES) {
                if (j >= NC && !wait(raw_free(v, st), (uint32_t)turn_st, 52)) break;
            } else if (j >= NS) {
                if (!wait_stage(v, j)) break;
                if (!v && j - NS + 1 == begins_q && begins_q < steps) load_queries();
            }
            if (j >= steps) continue;
            if (left == 0) {   // this share's part of another tile
                table = p.c.table + (long long)at.plan.b0 * p.c.pages_per_seq;
                pos = at.step * kPrefixStep + r;
                end = loads ? at.plan.prefix : 0;
                head_rows = at.head << p.c.page_shift;
                if (pos < end) page = table[pos >> p.c.page_shift];
                left = part(at);
            }
            int row = absent;
            if (pos < end) {
                if ((unsigned)page < (unsigned)p.c.n_pages) row = page * page_rows + head_rows + (pos & page_mask);   // (the host has seen that rows are 32-bit numbers)
                else if (!v && half == 0) paged_complain(p.c);
            }
            if (!NNC_BC(row >= 0 && row <= absent, 3601)) row = absent;
            if constexpr (CODES) {
                const uint32_t bar = raw_full(v, st), scales = raw_scales(v, st) + (uint32_t)r;
                if (loads && half == 1) {
                    if (row != absent) expect_more(bar, (uint32_t)p.box);
                    else {
                        for (int i = 0; i < p.box; i += 16) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(scales + i), "r"(0u) : "memory");
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // a later copy writes here, too
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_expect_tx(bar, T::kCodes);
                __syncwarp();
                if (loads && half == 0) tma_load_2d(raw_tile(v, st) + (uint32_t)(r * D), map, bar, 0, row);
                if (loads && half == 1 && row != absent) bulk_load(scales, (v ? p.c.v_scale : p.c.k_scale) + row, (uint32_t)p.box, bar);
            } else {
                const uint32_t bar = v ? v_full(st) : k_full(st);
                if (lane == 0) mbar_expect_tx(bar, T::kKV);
                __syncwarp();
                if (loads) tma_load_2d((v ? v_tile(st) : k_tile(st)) + (uint32_t)(half * T::kSlabKV + r * 128), map, bar, 64 * half, row);
            }
            pos += kPrefixStep;
            --left;
            if (left > 0 && pos < end) page = table[pos >> p.c.page_shift];   // on its way while this warp waits for the next stage
            if (++st == (CODES ? NC : NS)) { st = 0; turn_st ^= 1; }
        }
    } else if (CODES && warp >= 4 + 4 * kTeams) {   // ---------------- codes to bf16 rows: two warps for the keys of even steps, two for those of odd ones; the same for values ----------------
        const bool v = warp >= 8 + 4 * kTeams;
        constexpr int kPieces = D / 16, kRowsAtOnce = 32 / kPieces;   // a row is so many lanes' 16 codes
        const int piece = lane % kPieces, r0 = (warp & 1) * 32 + lane / kPieces;
        for (int j = warp >> 1 & 1; j < steps; j += 2) {
            const int st = j % NS, raw = j % NC;
            if (!wait(raw_full(v, raw), (uint32_t)(j / NC & 1), 53)) break;
            if (j >= NS && !wait_stage(v, j)) break;
            const uint32_t from = raw_tile(v, raw) + (uint32_t)(r0 * D + piece * 16), scales = raw_scales(v, raw) + (uint32_t)r0, tile = v ? v_tile(st) : k_tile(st);
#pragma unroll 2
            for (int i = 0; i < 32; i += kRowsAtOnce) {
                uint32_t x[4], byte, y[8];
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from + (uint32_t)(i * D)));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte) : "r"(scales + (uint32_t)i));
                const float scale = scale_from_byte(byte);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t h = e4m3x2_to_f16x2(x[e >> 1] >> (16 * (e & 1)) & 0xffffu);
                    const float2 f = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2 *>(&h)), make_float2(scale, scale));
                    y[e] = __byte_perm(__float_as_uint(f.x), __float_as_uint(f.y), 0x7632);   // the upper halves: the lower ones are 0
                }
                const int row = r0 + i;
#pragma unroll
                for (int e = 0; e < 2; ++e) {   // 16-byte chunks; lanes of the second slab in the other order, for other banks
                    const int which = e ^ (piece >> 2 & 1), chunk = 2 * piece + which;
                    const uint32_t dst = tile + (uint32_t)((chunk >> 3) * T::kSlabKV + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(which ? y[4] : y[0]), "r"(which ? y[5] : y[1]), "r"(which ? y[6] : y[2]), "r"(which ? y[7] : y[3]) : "memory");
                }
            }
            mbar_arrive(raw_free(v, raw));
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // generic-proxy writes, async-proxy (MMA) reads
            mbar_arrive(v ? v_full(st) : k_full(st));
        }
    } else if (warp <= 3) {   // ---------------- MMA issuers: scores; outputs ----------------
        const bool one = lane == 0;
        auto stage = [&](uint64_t desc, int st) { return desc + (uint64_t)((st * 2 * T::kKV) >> 4); };
        int st = 0, turn_st = 0;
        if (warp == 2) {
            constexpr uint32_t idesc = make_idesc(kPrefixStep, !BF, false);
            const uint64_t dq = make_smem_desc(q_tile), dk = make_smem_desc(k_tile(0));
            for (int j = 0, left = 0, tiles = 0; j < steps; ++j) {
                if (left == 0) {   // a new tile's queries
                    left = part(at);
                    if constexpr (CODES) {
                        if (j > 0 && !wait(s_full(j - 1), turn(j - 1), 54)) break;
                        load_queries();
                    }
                    if (!wait(q_ready, (uint32_t)(tiles & 1), 43)) break;
                    ++tiles;
                }
                --left;
                if (!wait(k_full(st), (uint32_t)turn_st, 44)) break;
                // the score buffer holds the probabilities of the step that had it before until their product is complete
                if (j >= kScoreBuffers && !wait(pv_done(j), turn(j) ^ 1u, 45)) break;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)     // 16 elements per instruction
                    mma_ss(one, tmem_base + kColS + (uint32_t)(j % kScoreBuffers * kPrefixStep), dq + (uint64_t)(((ks >> 2) * T::kQSlab + (ks & 3) * 32) >> 4),
                           stage(dk, st) + (uint64_t)(((ks >> 2) * T::kSlabKV + (ks & 3) * 32) >> 4), idesc, ks != 0);
                mma_commit(one, s_full(j));
                if (++st == NS) { st = 0; turn_st ^= 1; }
            }
        } else {
            constexpr uint32_t idesc = make_idesc(D, !BF, true);
            const uint64_t dv = make_smem_desc_mn(v_tile(0), T::kSlabKV);
            for (int j = 0, left = 0, nth = 0, team = 0; j < steps; ++j) {
                if (left == 0) { left = part(at); nth = 0; }
                const bool begins = nth < kTeams;   // the accumulator of this step's team is empty
                --left;
                ++nth;
                if (!wait(v_full(st), (uint32_t)turn_st, 47)) break;
                if (!wait(p_full(j), turn(j), 46)) break;
                tc_fence_after();
                const uint32_t pa = tmem_base + kColS + (uint32_t)(j % kScoreBuffers * kPrefixStep);   // two positions per column: first terms, then second ones
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                    for (int ks = 0; ks < kPrefixStep / 16; ++ks)
                        mma_ts(one, tmem_base + kColO + (uint32_t)(team * D), pa + (uint32_t)(kHeld == 1 ? (ks >> 1) * 32 + term * 16 + (ks & 1) * 8 : term * 32 + ks * 8), stage(dv, st) + (uint64_t)(ks * (2048 >> 4)), idesc,
                               !begins || term != 0 || ks != 0);
                mma_commit(one, pv_done(j));
                if (++team == kTeams) team = 0;
                if (++st == NS) { st = 0; turn_st ^= 1; }
            }
        }
    } else {   // ---------------- softmax: a query row per thread ----------------
        const int team = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;   // quarter: of tensor memory's lanes, which this warp may touch
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16, to = tmem_base + lane_addr + kColO + (uint32_t)(team * D);
        const int member = r / p.group, head_row = r - member * p.group;
        bool ok = true;
        // a barrier of all softmax warps that tells all of them whether any has seen something
        auto any_of_all = [&](bool mine) -> bool {
            uint32_t any;
            __syncwarp();
            asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbarrier.cta.red.or.aligned.pred p, 1, %2, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(any) : "r"((uint32_t)mine), "n"(128 * kTeams) : "memory");
            return any != 0u;
        };
        // Where a wait gave up, a warp still comes to the barriers below, once for every part of a tile, so that no other waits there for it
        for (int j0 = 0; j0 < steps;) {
            const int n = (int)min((long long)(at.plan.steps - at.step), t1 - at.index), s0 = at.step;   // this share's part of a tile: steps j0 .. j0 + n - 1
            const int nth = at.tile * p.per_tile + member;
            const bool valid = member < p.per_tile && nth < at.plan.members && takes_prefix(at.plan.prefix, p.lens[at.plan.b0 + nth]);
            const bool idle = !__any_sync(0xffffffffu, valid);   // no query of this warp counts
            // pages that the pool does not have: a lane's 16 positions of a step, looked up a step ahead
            auto has_page = [&](int i) {
                const int pos = (s0 + i) * kPrefixStep + 16 * (lane & 3);
                return i >= n || pos >= at.plan.prefix || (unsigned)p.c.table[(long long)at.plan.b0 * p.c.pages_per_seq + (pos >> p.c.page_shift)] < (unsigned)p.c.n_pages;
            };
            const int first = (team + kTeams - j0 % kTeams) % kTeams;   // this team's first step
            bool has = has_page(first);
            float m_used = -INFINITY, l = 0.f, ref = 0.f;
            // The first time once without effect, while rows and queries are on their way, on the empty accumulator instead of scores: fetching the
            // instructions of a step takes longer than the step
            for (int i = j0 == 0 ? first - kTeams : first; ok && i < n; i += kTeams) {
                const int j = j0 + i, p0 = (s0 + i) * kPrefixStep;
                const bool dry = i < first;
                if (!dry) ok = __all_sync(0xffffffffu, mbar_wait(s_full(j), turn(j), abort_flag, p.wait_status, 48));
                if (!ok) break;
                tc_fence_after();
                const uint32_t there = __ballot_sync(0xffffffffu, has) & 0xfu;   // per 16 positions
                if (!dry) has = has_page(i + kTeams);
                if (idle) {   // (its rows of P are whatever the scores' bits are, and nobody's)
                    if (!dry) mbar_arrive(p_full(j));
                    continue;
                }
                const uint32_t ts = dry ? to : tmem_base + lane_addr + kColS + (uint32_t)(j % kScoreBuffers * kPrefixStep);
                uint32_t held[kHeld][32];
                auto fetch = [&](int c0) {   // columns from 32 c0 on
#pragma unroll
                    for (int c = 0; c < kHeld; ++c) tmem_ld32_nowait(ts + 32u * (c0 + c), held[c]);
                    tmem_wait_ld();
                    if (p.flip) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
#pragma unroll
                            for (int c = 0; c < kHeld; ++c) held[c][e] ^= p.flip;
                    }
                    if (p0 + kPrefixStep > at.plan.prefix || there != 0xfu) {
#pragma unroll
                        for (int c = 0; c < kHeld; ++c)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (p0 + 32 * (c0 + c) + e >= at.plan.prefix || !(there >> (2 * (c0 + c) + e / 16) & 1u)) held[c][e] = 0xff800000u;   // -infinity
                    }
                };
                if constexpr (kHeld == 2) fetch(0);
                auto scores_of = [&](int c) -> const uint32_t (&)[32] {
                    if constexpr (kHeld == 1) fetch(c);
                    return held[c & (kHeld - 1)];
                };
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll kHeld
                for (int c = 0; c < 2; ++c) {
                    const auto &x = scores_of(c);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) mx[e / 2 & 3] = top3(mx[e / 2 & 3], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                }
                const float m_step = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
                if (i <= first) {
                    m_used = m_step;
                    l = 0.f;
                } else {
                    // the maximum that O refers to moves only when a step passes it by 2^8
                    const bool need = valid && m_step > m_used + kLazyMax;
                    if (__any_sync(0xffffffffu, need)) {
                        ok = __all_sync(0xffffffffu, mbar_wait(pv_done(j - kTeams), turn(j - kTeams), abort_flag, p.wait_status, 49));
                        if (!ok) break;
                        tc_fence_after();
                        const float m_new = need ? m_step : m_used;
                        const float alpha = need ? ex2_approx(m_used - m_new) : 1.f;
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t t[32];
                            tmem_ld32(to + 32u * c, t);
#pragma unroll
                            for (int e = 0; e < 32; ++e) t[e] = __float_as_uint(__uint_as_float(t[e]) * alpha);
                            tmem_st32(to + 32u * c, t);
                        }
                        tmem_wait_st();
                        l *= alpha;
                        m_used = m_new;
                    }
                }
                ref = (m_used == -INFINITY ? 0.f : m_used) - kLift;   // nothing attended so far: every weight is 0
                const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), neg = make_float2(-ref, -ref);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll kHeld
                for (int c = 0; c < 2; ++c) {
                    uint32_t hi[16], lo[16];
                    const auto &sv = scores_of(c);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1])), scale2, neg);
                        const float2 w = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        sum[e & 1] = __fadd2_rn(sum[e & 1], w);
                        if constexpr (BF) {
                            hi[e] = round_bf16x2(w.x, w.y);
                            lo[e] = round_bf16x2(w.x - bf16_lo(hi[e]), w.y - bf16_hi(hi[e]));
                        } else {
                            const __half2 a = __floats2half2_rn(w.x, w.y);
                            const float2 f = __half22float2(a);
                            const __half2 b = __floats2half2_rn(w.x - f.x, w.y - f.y);
                            hi[e] = *reinterpret_cast<const uint32_t *>(&a);
                            lo[e] = *reinterpret_cast<const uint32_t *>(&b);
                        }
                    }
                    tmem_st16(ts + (kHeld == 1 ? 32u : 16u) * c, hi);
                    tmem_st16(ts + (kHeld == 1 ? 32u * c + 16u : 32u + 16u * c), lo);
                }
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                tmem_wait_st();
                tc_fence_before();
                if (!dry) mbar_arrive(p_full(j));
            }
            // ---- the part is done: two teams write half of the columns of the accumulators' sum each ----
            if (first >= n) { m_used = -INFINITY; l = 0.f; }   // no step of this team's
            const float2 x = make_float2(m_used == -INFINITY && l == 0.f ? -INFINITY : ref, l);
            ml_s[team][r] = x;
            asm volatile("bar.sync 1, %0;" ::"n"(128 * kTeams) : "memory");
            const int last = j0 + n - 1;   // its product is complete when all before it are
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(pv_done(last), turn(last), abort_flag, p.wait_status, 50));
            constexpr int kWriters = 2;   // teams, each half of the columns
            const long long row = (long long)at.plan.b0 * p.n_q + ((long long)at.head * at.plan.members + nth) * p.group + head_row + kPrefixRows * cta;
            const bool store = ok && valid && team < kWriters && NNC_BC(row < p.part_rows, 3602);
            bool odd = false;   // a sum is no number, although the weights' is
            if (ok && !idle && team < kWriters) {
                tc_fence_after();
                float2 of[kTeams];
                float m = -INFINITY, sum = 0.f, weight[kTeams];
#pragma unroll
                for (int t = 0; t < kTeams; ++t) {
                    of[t] = ml_s[t][r];
                    m = fmaxf(m, of[t].x);
                }
#pragma unroll
                for (int t = 0; t < kTeams; ++t) {
                    weight[t] = exp2f(of[t].x - (m == -INFINITY ? 0.f : m));
                    sum = fmaf(weight[t], of[t].y, sum);
                }
                if (store && team == 0) p.s.ml[row] = make_float2(m, sum);
                const uint32_t from = tmem_base + lane_addr + kColO + (uint32_t)(team * (D / kWriters));
                float4 *dst = p.s.o + (team * (D / (4 * kWriters))) * p.part_rows + row;
                float all_sums = 0.f;
#pragma unroll 1
                for (int c = 0; c < D / (16 * kWriters); ++c) {   // 16 columns at a time
                    uint32_t u[kTeams][16];
#pragma unroll
                    for (int t = 0; t < kTeams; ++t) tmem_ld16_nowait(from + (uint32_t)(t * D + 16 * c), u[t]);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float v = 0.f;
#pragma unroll
                        for (int t = 0; t < kTeams; ++t)   // (an accumulator that no step of this part wrote holds anything)
                            if ((t + kTeams - j0 % kTeams) % kTeams < n) v = fmaf(weight[t], __uint_as_float(u[t][e]), v);
                        u[0][e] = __float_as_uint(v);
                        if constexpr (!CODES) all_sums += v;
                    }
                    if (store) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store16(dst + (4 * c + e) * p.part_rows, u[0] + 4 * e);
                    }
                }
                if constexpr (!CODES) odd = store && !(fabsf(all_sums) < INFINITY) && sum == sum;
                tc_fence_before();
            }
            // A column of values with an infinity in an attended row is that infinity, however small the row's weight (two of different signs,
            // or NaN, leave no number).  The products cannot say so: a weight's lower term is of either sign or 0, and 0 times infinity is NaN.  So a
            // part whose sums are not all finite looks through its value rows again, a row's 16-byte pieces on neighbouring lanes.  Not for rows whose
            // weights' sum is itself no number, which their results then are, too; and not of codes, which are never infinite.
            // From this barrier on the accumulators and ml_s are free.
            if constexpr (CODES) asm volatile("bar.sync 1, %0;" ::"n"(128 * kTeams) : "memory");
            else if (any_of_all(odd)) {
                constexpr int kSoft = 128 * kTeams, kPieces = D / 8;
                const int t = tid - 128;
                if (t < D) odd_s[t] = 0u;
                any_of_all(false);
                uint32_t plus = 0, minus = 0, none = 0;   // a bit per column of this lane's piece
                const int piece = t % kPieces, end = min((s0 + n) * kPrefixStep, at.plan.prefix);
                const int32_t *const table = p.c.table + (long long)at.plan.b0 * p.c.pages_per_seq;
#pragma unroll 4
                for (int pos = s0 * kPrefixStep + t / kPieces; pos < end; pos += kSoft / kPieces) {
                    const int page = table[pos >> p.c.page_shift];
                    if ((unsigned)page >= (unsigned)p.c.n_pages) continue;
                    const uint4 v = *reinterpret_cast<const uint4 *>(p.c.v + paged_row(p.c, page, at.head, pos & ((1 << p.c.page_shift) - 1)) * (2 * D) + 16 * piece);
                    const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
                        const uint32_t x = words[e / 2] >> (16 * (e & 1)) & 0xffffu, size = x & 0x7fffu;
                        if (size >= kInf) (size > kInf ? none : x == size ? plus : minus) |= 1u << e;
                    }
                }
                if (plus | minus | none)
#pragma unroll 1
                    for (int e = 0; e < 8; ++e)
                        if (const uint32_t bits = (plus >> e & 1u) | (minus >> e & 1u) << 1 | (none >> e & 1u) << 2) atomicOr(&odd_s[8 * piece + e], bits);
                any_of_all(false);
                if (store) {
#pragma unroll 1
                    for (int c = 0; c < D / kWriters; ++c) {
                        const int col = team * (D / kWriters) + c;
                        const uint32_t bits = odd_s[col];
                        if (bits) reinterpret_cast<float *>(p.s.o + (col >> 2) * p.part_rows + row)[col & 3] = bits == 1u ? INFINITY : bits == 2u ? -INFINITY : __uint_as_float(0x7fffffffu);
                    }
                    if (team == 0 && p.s.ml[row].x == -INFINITY) p.s.ml[row].x = kNothing;
                }
                any_of_all(false);
            }
            j0 += n;
            at.index += n - 1;
            at.step += n - 1;
            advance(p, at);
        }
    }

    // ---- teardown ----
    __syncwarp();
    if (*abort_flag && tid == 0) {   // let copies that are still in flight land before the shared memory is released
        const unsigned long long since = global_ns();
        while (global_ns() - since < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemColumns) : "memory");
}

// ---- joining: a CTA a (sequence, KV head) -------------------------------------------------------------------------------------
//
// Its query heads' rows are neighbours in every piece.  A thread takes four elements of a row of every kth piece, as a softmax of its own, and
// those that share a row's elements are joined in shared memory: so what a CTA loads after its sequence's record depends on that alone.  Bound by that
// chain: 9 us for 64 sequences of 32 heads in 10 pieces (11 MB).

constexpr int kJoinThreads = 256;

struct JoinParams {
    PrefixScratch s;
    char *out;
    float *lse;
    long long out_stride, part_rows;
    int n_kv, group, n_q;
};

template <int D, bool BF, bool CODES>   // BF: results are bf16, otherwise fp16; the cache's type, or codes
__global__ void __launch_bounds__(kJoinThreads) attn_prefix_join_kernel(const JoinParams p) {
    constexpr int kFours = D / 4, kRows = kJoinThreads / kFours;   // of a row; rows at a time
    __shared__ float4 sums[kJoinThreads];
    __shared__ float2 mls[kJoinThreads];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, b = blockIdx.x / p.n_kv, head = blockIdx.x - b * p.n_kv;
    const PrefixOf of = p.s.of[b];
    long long first_row = 0;
    int n = 0;
    if (of.steps) {
        const long long lo = of.first + (long long)head * of.per_head, c_lo = lo / of.share;
        n = (int)((lo + of.steps - 1) / of.share - c_lo) + 1;
        first_row = of.row + (long long)head * of.rows_per_head + kPrefixRows * c_lo;
        if (!NNC_BC(first_row >= 0 && first_row + (long long)kPrefixRows * (n - 1) + p.group <= p.part_rows, 3603)) n = 0;
    }
    for (int h0 = 0; h0 < p.group; h0 += kRows) {
        const int rows = min(kRows, p.group - h0);
        const long long q_row = (long long)b * p.n_q + (long long)head * p.group + h0;
        // thread: elements c4 of row h, pieces k, k + apart, ..
        const int items = rows * kFours, apart = kJoinThreads / items, item = tid % items, k = tid / items, h = item % rows, c4 = item / rows;
        const bool mine = k < apart;
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](float2 ml, float4 v) {
            if (ml.x == -INFINITY) return;
            const float top = fmaxf(m, ml.x), a = exp2f(m - top), w = exp2f(ml.x - top);
            m = top;
            l = fmaf(l, a, ml.y * w);
            o.x = fmaf(o.x, a, v.x * w); o.y = fmaf(o.y, a, v.y * w); o.z = fmaf(o.z, a, v.z * w); o.w = fmaf(o.w, a, v.w * w);
        };
        const float2 *ml = p.s.ml + first_row + h0 + h;
        const float4 *src = p.s.o + c4 * p.part_rows + first_row + h0 + h;
        float2 tail_ml = make_float2(-INFINITY, 0.f);
        float4 tail = o;
        if (mine) {
            constexpr int kAhead = 8;   // pieces on their way at a time
            if (k == 0) {
                tail_ml = p.s.tail_ml[q_row + h];
                tail = *reinterpret_cast<const float4 *>(p.s.tail + (q_row + h) * D + 4 * c4);
                if (!CODES && tail_ml.x == -INFINITY && !(fabsf((tail.x + tail.y) + (tail.z + tail.w)) < INFINITY)) tail_ml = make_float2(kNothing, 0.f);
            }
            for (int i0 = k; i0 < n; i0 += kAhead * apart) {
                float2 x[kAhead];
                float4 v[kAhead];
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
                    if (i0 + a * apart < n) {
                        x[a] = ml[(long long)kPrefixRows * (i0 + a * apart)];
                        v[a] = src[(long long)kPrefixRows * (i0 + a * apart)];
                    }
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
                    if (i0 + a * apart < n) add(x[a], v[a]);
            }
            add(tail_ml, tail);
        }
        if (apart > 1) {
            sums[tid] = o;
            mls[tid] = make_float2(m, l);
            __syncthreads();
            if (mine && k == 0)
                for (int j = 1; j < apart; ++j) add(mls[item + j * items], sums[item + j * items]);
        }
        const bool store = mine && k == 0;
        if constexpr (!CODES)
            if (store && l == l && !(fabsf((o.x + o.y) + (o.z + o.w)) < INFINITY)) {
                // An infinite sum is its column's result, whatever it weighs (0 times it is no number): such columns once more, with the weights known
                float4 again = make_float4(0.f, 0.f, 0.f, 0.f);
                auto sum = [](float w, float v, float sum) { return fabsf(v) == INFINITY ? sum + v : fmaf(w, v, sum); };
                auto weigh = [&](float x, float4 v) {
                    const float w = m == -INFINITY ? 0.f : exp2f(x - m);
                    again.x = sum(w, v.x, again.x); again.y = sum(w, v.y, again.y); again.z = sum(w, v.z, again.z); again.w = sum(w, v.w, again.w);
                };
#pragma unroll 4
                for (int i = 0; i < n; ++i) weigh(ml[(long long)kPrefixRows * i].x, src[(long long)kPrefixRows * i]);
                weigh(tail_ml.x, tail);
                if (!(fabsf(o.x) < INFINITY)) o.x = again.x;
                if (!(fabsf(o.y) < INFINITY)) o.y = again.y;
                if (!(fabsf(o.z) < INFINITY)) o.z = again.z;
                if (!(fabsf(o.w) < INFINITY)) o.w = again.w;
            }
        if (store) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const long long at = b * p.out_stride + ((long long)head * p.group + h0 + h) * D + 4 * c4;
            uint2 v;
            if constexpr (BF) v = make_uint2(round_bf16x2(o.x * inv, o.y * inv), round_bf16x2(o.z * inv, o.w * inv));
            else {
                const __half2 lo = __floats2half2_rn(o.x * inv, o.y * inv), hi = __floats2half2_rn(o.z * inv, o.w * inv);
                v = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
            }
            *reinterpret_cast<uint2 *>(p.out + at * 2) = v;
            if (p.lse && c4 == 0) p.lse[q_row + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
        __syncthreads();
    }
}

size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

// behind the tail's own scratch
PrefixScratch carve(char *at, int batch, int n_q, int d, long long part_rows, size_t *bytes) {
    size_t used = 0;
    auto take = [&](size_t n) { char *p = at + used; used += aligned(n); return p; };
    PrefixScratch s;
    s.plan = (PrefixPlan *)take(sizeof(PrefixPlan) * batch);
    s.of = (PrefixOf *)take(sizeof(PrefixOf) * batch);
    s.ml = (float2 *)take(8 * part_rows);
    s.o = (float4 *)take(4 * part_rows * d);
    s.tail_ml = (float2 *)take(8ll * batch * n_q);
    s.tail = (float *)take(4ll * batch * n_q * d);
    if (bytes) *bytes = used;
    return s;
}
long long part_rows_of(int batch, int n_q) { return (long long)batch * n_q + (long long)kPrefixRows * kPrefixMaxCtas; }

// the pool of one kind as rows of a KV head's positions
bool make_pool_map(CUtensorMap *map, const nnc_paged_kv &c, const void *pool, int box) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const bool codes = c.type == NNC_E4M3;
    const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.n_pages * c.n_kv_heads * c.page_size}, strides[1] = {(cuuint64_t)c.head_dim * (codes ? 1 : 2)};
    const cuuint32_t boxes[2] = {codes ? (cuuint32_t)c.head_dim : 64u, (cuuint32_t)box}, one[2] = {1, 1};
    return enc(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : c.type == NNC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(pool), dims, strides, boxes, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, codes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the queries: [sequence][head][element], in boxes of a tile's
bool make_query_map(CUtensorMap *map, const void *q, bool bf, int d, int n_q, int batch, int64_t stride, int group, int per_tile) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)n_q, (cuuint64_t)batch}, strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)stride * 2};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)group, (cuuint32_t)per_tile}, one[3] = {1, 1, 1};
    return enc(map, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(q), dims, strides, boxes, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int KV> cudaError_t launch_prefix_of(const LaunchCtx &lc, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PrefixParams &p) {
    typedef Tiles<D, KV == NNC_E4M3> T;
    static unsigned long long raised = 0;
    auto kern = attn_prefix_kernel<D, KV>;
    if (cudaError_t e = ensure_dynamic_smem(kern, T::kSmem, &raised); e != cudaSuccess) return e;
    const int ctas = lc.sm_count < kPrefixMaxCtas ? lc.sm_count : kPrefixMaxCtas;
    return launch_smem(lc, kern, dim3((unsigned)ctas), dim3(T::kThreads), (size_t)T::kSmem, mq, mk, mv, p);
}
template <int D> cudaError_t launch_prefix_typed(const LaunchCtx &lc, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PrefixParams &p, int kv) {
    return kv == NNC_BF16 ? launch_prefix_of<D, NNC_BF16>(lc, mq, mk, mv, p) : kv == NNC_F16 ? launch_prefix_of<D, NNC_F16>(lc, mq, mk, mv, p) : launch_prefix_of<D, NNC_E4M3>(lc, mq, mk, mv, p);
}

template <int D> cudaError_t launch_join_of(const LaunchCtx &lc, const JoinParams &p, int kv, long long ctas) {
    const dim3 grid((unsigned)ctas), block(kJoinThreads);
    if (kv == NNC_BF16) return launch(lc, attn_prefix_join_kernel<D, true, false>, grid, block, p);
    if (kv == NNC_F16) return launch(lc, attn_prefix_join_kernel<D, false, false>, grid, block, p);
    return launch(lc, attn_prefix_join_kernel<D, true, true>, grid, block, p);
}

}  // namespace

size_t attn_prefix_scratch_bytes(int batch, int n_q_heads, int head_dim) {
    size_t bytes = 0;
    carve(nullptr, batch, n_q_heads, head_dim, part_rows_of(batch, n_q_heads), &bytes);
    return NNC_ATTN_PAGED_SCRATCH_BYTES + bytes;
}

cudaError_t launch_attn_prefix(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, const int32_t *starts,
                               const int32_t *shared, int n_groups, void *out, float *lse, int type, int batch, int n_q_heads, int64_t q_stride,
                               int64_t out_stride, float scale, void *scratch) {
    // Every sequence's own rows, the shared ones among them: fp32; fp16 queries of codes, as the codes' operand is bf16 here and both operands of a product have one
    // type; more query heads than a tile has rows, which share rows among themselves; queries whose rows overlap, which a tensor map does not describe; one sequence.  And small batches: reading all of a table's
    // rows for each sequence, mostly from L2, goes at some 10 TB/s per eight query heads behind 9 us, three launches take 17 to 25 us.  Both
    // sides, us (three launches first), 4 query heads of 128 and 12 of 64 per KV head: 35 MB 19 and 15, 135 MB 27.6 and 27.6, 140 MB 26.0 and
    // 24.5, 155 MB 27.7 and 25.8, 540 MB 32 and 64; 34 MB 31 and 17, 70 MB 23.3 and 25.0, 78 MB 29 and 27, 270 MB 37 and 58.  Codes:
    // 135 MB 35 and 34, 270 MB 38 and 52; 12 of 64, 135 MB 40 and 54.  (Lengths are the device's: three of 500 under a table for 65536 take three launches, 12.8
    // us instead of 8.4.)
    const int eights = (n_q_heads / cache.n_kv_heads + 7) / 8;
    const double rows_bytes = (cache.type == NNC_E4M3 ? 2.0 : 4.0) * batch * cache.pages_per_seq * cache.page_size * cache.n_kv_heads * cache.head_dim;
    if (type == NNC_F32 || (cache.type == NNC_E4M3 && type != NNC_BF16) || n_q_heads / cache.n_kv_heads > kPrefixRows || (batch > 1 && q_stride < (int64_t)n_q_heads * cache.head_dim) ||
        batch == 1 || rows_bytes * eights < 140e6)
        return launch_attn_paged(lc, q, cache, lens, out, lse, type, batch, n_q_heads, q_stride, out_stride, scale, 0, scratch, NNC_ATTN_PAGED_SCRATCH_BYTES);
    if (!attn_tail_fits(cache, batch)) return cudaErrorInvalidValue;
    const int d = cache.head_dim, group = n_q_heads / cache.n_kv_heads;
    const bool bf = type == NNC_BF16;
    const PrefixScratch s = carve((char *)scratch + NNC_ATTN_PAGED_SCRATCH_BYTES, batch, n_q_heads, d, part_rows_of(batch, n_q_heads), nullptr);
    // Groups of few sequences read their own rows, through the kernel for what lies behind prefixes.  How many a group has is known to the device alone
    // (n_groups may count groups of none, so that a captured call has room for them).  us, prefix of 8192 or 16384 at once / each its own: one sequence of
    // 4 heads 191 / 177, of 16 81 / 68 and 64 / 43, of 24 85 / 97 and 60 / 58, of 32 92 / 108 and 65 / 65; two of 4 108 / 182, of 8 with heads of 64 86 / 95.
    // Codes: one of 32 103 / 88 and 80 / 57, of 64 86 / 89 and 63 / 60; two of 4 140 / 106, of 16 61 / 54, of 24 62 / 79 and 52 / 54; three of 4 102 / 100,
    // of 16 52 / 52; four of 4 88 / 105, of 8 with heads of 64 72 / 72.  Where no group has as many, three launches do what one would: 192 instead of 184 us
    // for 32 of 8192, codes 115 instead of 106.
    const int least = cache.type == NNC_E4M3 ? (group >= 48 ? 1 : group >= 24 ? 2 : group >= 16 ? 3 : 4) : group >= 32 ? 1 : 2;
    const PrefixGroups groups{starts, shared, n_groups, batch, least};
    PrefixParams p = {};
    p.c = paged_view(cache, lc.status);
    p.groups = groups;
    p.s = s;
    p.lens = lens;
    p.part_rows = part_rows_of(batch, n_q_heads);
    p.group = group; p.per_tile = kPrefixRows / group; p.n_q = n_q_heads;
    p.box = cache.page_size < kPrefixStep ? cache.page_size : kPrefixStep;
    p.flip = scale < 0.f ? 0x80000000u : 0u;
    p.scale_log2 = fabsf(scale) * 1.4426950408889634f;
    if (p.scale_log2 == 0.f) p.scale_log2 = 1e-45f;   // (0 times the -infinity of a masked score would be no number)
    p.wait_status = lc.status - 1;                    // the tensor-core kernels' word lies before the paged-cache kernels'
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, q, bf, d, n_q_heads, batch, batch > 1 ? q_stride : (int64_t)n_q_heads * d, group, p.per_tile)) return cudaErrorUnknown;
    if (!make_pool_map(&mk, cache, cache.k, p.box) || !make_pool_map(&mv, cache, cache.v, p.box)) return cudaErrorUnknown;
    LaunchCtx early = lc;
    early.pdl = true;
    cudaError_t e = d == 64 ? launch_prefix_typed<64>(early, mq, mk, mv, p, cache.type) : launch_prefix_typed<128>(early, mq, mk, mv, p, cache.type);
    if (e != cudaSuccess) return e;
    e = launch_attn_tail(lc, q, cache, lens, groups, s.tail, s.tail_ml, type, n_q_heads, q_stride, scale, scratch, NNC_ATTN_PAGED_SCRATCH_BYTES);
    if (e != cudaSuccess) return e;
    JoinParams j = {};
    j.s = s; j.out = (char *)out; j.lse = lse; j.out_stride = out_stride; j.part_rows = p.part_rows;
    j.n_kv = cache.n_kv_heads; j.group = group; j.n_q = n_q_heads;
    const long long ctas = (long long)batch * cache.n_kv_heads;
    return d == 64 ? launch_join_of<64>(early, j, cache.type, ctas) : launch_join_of<128>(early, j, cache.type, ctas);
}

}  // namespace nnc
