// Attention of one new token per sequence where groups of sequences share the first positions of a paged cache: the shared rows are read
// once for the whole group.
//
//   s_n = scale q.k_n,  o = sum_n exp(s_n - m) v_n / sum_n exp(s_n - m),  n < lens[b], in three launches:
//   prefix   (this file)  m, l = sum exp(s_n - m), o~ = sum exp(s_n - m) v_n over the shared positions, for all queries of a group at a time
//   tail     (attn_prefix_tail.cu)  the same, divided, over what lies behind them, sequence by sequence
//   joining  (this file)  both, weighed by their sums
//
// The queries of a group's sequences for one KV head are rows of one operand, so the prefix is a pair of matrix products with up to 128
// rows, and tcgen05 does them: S = Q K^T and O += P V with S, P and O in tensor memory, K and V pages fetched by TMA (a page of a KV head is a
// [page_size][head_dim] matrix; boxes of 16 to 64 positions, zeros where a page is missing).  Bound by reading the prefix where a group
// fills one tile, by the exponentials where it fills several.
//   - The list of (group, KV head, tile, step of 64 positions) is cut into one contiguous share per CTA; the groups' lengths live on the
//     device, so every CTA adds up the list itself.  A share may begin and end inside a tile.
//   - Two CTAs of 192 threads per SM: TMA producer, MMA issuer, four softmax warps with a query row per thread, as in attn_prefill_f16.cu:
//     two score buffers, so that the products of the next step run while the softmax works on this one.
//   - Queries enter exactly.  Probabilities are two terms of the cache's type (bf16: 16 bits, fp16: 22), written over the scores they
//     come from: one bf16 term alone would add an error of the size of the result's own rounding.  fp32 queries and results would need three
//     terms and shorter sums; they go through the kernel that reads every sequence's rows.
#include <cuda_fp16.h>

#include "attn_prefill_common.cuh"
#include "attn_prefix.cuh"

namespace nnc {

namespace {

constexpr int kThreads = 192;
constexpr int kSoftmaxRows = 128;
constexpr uint32_t kColS = 0, kColO = 128, kTmemColumns = 256;   // score buffers at columns 0 and 64
constexpr float kLn2 = 0.69314718055994530942f;

template <int D> struct Tiles {
    static constexpr int kHalves = D / 64;                        // slabs of 64 elements
    static constexpr int kQSlab = kPrefixRows * 128, kQ = kHalves * kQSlab;
    static constexpr int kSlabKV = kPrefixStep * 128, kKV = kHalves * kSlabKV;
    static constexpr int kSmem = kQ + 4 * kKV + 1024 /*alignment*/ + 128 /*barriers*/;
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

// BF: bf16 caches, otherwise fp16; queries are of the cache's type
template <int D, bool BF>
__global__ void __launch_bounds__(kThreads, 2)
attn_prefix_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const PrefixParams p) {
    typedef Tiles<D> T;
    // fp16 probabilities are scaled by 2^6, so that small ones keep their bits (at most 2^8 by the lazy maximum: below 2^15; sums are scaled alike)
    constexpr float kLift = BF ? 0.f : 6.f;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_tile = base;
    auto k_tile = [&](int st) { return base + (uint32_t)(T::kQ + st * 2 * T::kKV); };
    auto v_tile = [&](int st) { return k_tile(st) + (uint32_t)T::kKV; };
    const uint32_t bars = base + (uint32_t)(T::kQ + 4 * T::kKV);
    const uint32_t q_ready = bars;
    auto k_full = [&](int st) { return bars + 8u * (1 + st); };
    auto v_full = [&](int st) { return bars + 8u * (3 + st); };
    auto s_full = [&](int st) { return bars + 8u * (5 + st); };
    auto p_full = [&](int st) { return bars + 8u * (7 + st); };
    auto pv_done = [&](int st) { return bars + 8u * (9 + st); };
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s, first_g;
    __shared__ long long first_rest, sums[kThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int *abort_flag = &abort_s;
    if (tid == 0) {
        abort_s = 0;
        mbar_init(q_ready, 1);
        for (int st = 0; st < 2; ++st) {
            mbar_init(k_full(st), 1); mbar_init(v_full(st), 1); mbar_init(s_full(st), 1);
            mbar_init(p_full(st), kSoftmaxRows); mbar_init(pv_done(st), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();   // groups, lengths, tables, queries and rows may be the preceding kernel's
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
    if (cta == 0) {   // for the joining kernel
        if (tid == 0) p.s.head->share = share;
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
    const uint32_t tmem_base = tmem_base_s;
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
    auto more = [&]() { return at.index < t1 && at.g < p.groups.n_groups; };

    if (warp == 0) {   // ---------------- TMA producer: a lane a box ----------------
        // Lane: kind (K or V), box of the step's positions, half of the head's elements.  Rows are looked up a step before K needs them, and V
        // takes K's.
        const int half = lane & 1, r = (lane >> 1 & 3) * p.box;
        const bool loads = lane < 16 && half < T::kHalves && r < kPrefixStep, is_v = lane >= 8;
        const int absent = (int)min(paged_rows(p.c), 0x7fffffffll);   // a row outside the tensor: zeros
        Step far = at;                                                // the step whose rows are looked up next
        auto look = [&]() {
            if (!(far.index < t1 && far.g < p.groups.n_groups)) return absent;
            const int pos = far.step * kPrefixStep + r;
            int page = -1;
            if (loads && pos < far.plan.prefix) {
                page = p.c.table[(long long)far.plan.b0 * p.c.pages_per_seq + (pos >> p.c.page_shift)];
                if ((unsigned)page >= (unsigned)p.c.n_pages) { page = -1; if (!is_v && half == 0) paged_complain(p.c); }
            }
            const long long row = page < 0 ? absent : paged_row(p.c, page, far.head, pos & ((1 << p.c.page_shift) - 1));
            advance(p, far);
            return NNC_BC(row >= 0 && row <= absent, 3601) ? (int)row : absent;
        };
        // The box of stage `st` for this kind; the other kind's lanes look on
        auto load = [&](bool v, int st, int row) {
            const uint32_t bar = v ? v_full(st) : k_full(st);
            if (lane == 0) mbar_expect_tx(bar, T::kKV);
            __syncwarp();
            if (loads && is_v == v) tma_load_2d((v ? v_tile(st) : k_tile(st)) + half * T::kSlabKV + r * 128, v ? &map_v : &map_k, bar, 64 * half, row);
        };
        auto load_queries = [&](const Step &x) {   // [sequence][query head of the KV head][64]: a row of the tile after the other
            if (lane == 0) mbar_expect_tx(q_ready, (uint32_t)(T::kHalves * p.per_tile * p.group * 128));
            __syncwarp();
            if (lane < T::kHalves) tma_load_3d(q_tile + lane * T::kQSlab, &map_q, q_ready, 64 * lane, x.head * p.group, x.plan.b0 + x.tile * p.per_tile);
        };
        long long steps = 0;   // of this share
        for (Step s = at; s.index < t1 && s.g < p.groups.n_groups;) {   // a tile's at a time
            const long long n = min((long long)(s.plan.steps - s.step), t1 - s.index);
            steps += n;
            s.index += n - 1;
            s.step += (int)n - 1;
            advance(p, s);
        }
        // A stage's K tile is free as soon as the S of the step that read it is complete: K_{j+1} is requested when S_{j-1} is
        // complete, V_j when O += P_{j-2} V_{j-2} is.
        int row0 = look(), row1 = look(), row2 = absent;   // of steps j, j + 1, j + 2
        if (steps > 0) {
            load_queries(at);
            load(false, 0, row0);
        }
        if (steps > 1) load(false, 1, row1);
        for (long long j = 0; j < steps; ++j) {
            const int st = (int)(j & 1);
            row2 = look();
            if (j >= 1) {
                if (!__all_sync(0xffffffffu, mbar_wait(s_full(st ^ 1), (uint32_t)(((j - 1) >> 1) & 1), abort_flag, p.wait_status, 41))) break;
                advance(p, at);
                if (at.step == 0) load_queries(at);   // a new tile's: the last one's have been multiplied for the last time
                if (j + 1 < steps) load(false, st ^ 1, row1);
            }
            if (j >= 2 && !__all_sync(0xffffffffu, mbar_wait(pv_done(st), (uint32_t)(((j - 2) >> 1) & 1), abort_flag, p.wait_status, 42))) break;
            load(true, st, row0);
            row0 = row1;
            row1 = row2;
        }
    } else if (warp == 1) {
        if (lane == 0) {   // ---------------- MMA issuer ----------------
            constexpr uint32_t idesc_qk = make_idesc(kPrefixStep, !BF, false), idesc_pv = make_idesc(D, !BF, true);
            const uint64_t dq = make_smem_desc(q_tile);
            const uint64_t dk[2] = {make_smem_desc(k_tile(0)), make_smem_desc(k_tile(1))};
            const uint64_t dv[2] = {make_smem_desc_mn(v_tile(0), T::kSlabKV), make_smem_desc_mn(v_tile(1), T::kSlabKV)};
            int pieces = 0;
            Step next = at;
            auto issue_qk = [&](int j) -> bool {
                const int st = j & 1, u = j >> 1;
                if (j == 0 || next.step == 0) {   // a new tile's queries
                    if (!mbar_wait(q_ready, (uint32_t)(pieces & 1), abort_flag, p.wait_status, 43)) return false;
                    ++pieces;
                }
                if (!mbar_wait(k_full(st), (uint32_t)(u & 1), abort_flag, p.wait_status, 44)) return false;
                // the score buffer holds P_{j-2} until O += P_{j-2} V_{j-2} has completed
                if (j >= 2 && !mbar_wait(pv_done(st), (uint32_t)((u - 1) & 1), abort_flag, p.wait_status, 45)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)     // 16 elements per instruction
                    umma_bf16(tmem_base + kColS + (uint32_t)st * kPrefixStep, dq + (uint64_t)(((ks >> 2) * T::kQSlab + (ks & 3) * 32) >> 4),
                              dk[st] + (uint64_t)(((ks >> 2) * T::kSlabKV + (ks & 3) * 32) >> 4), idesc_qk, ks != 0);
                umma_commit(s_full(st));
                advance(p, next);
                return true;
            };
            auto more_qk = [&]() { return next.index < t1 && next.g < p.groups.n_groups; };
            bool ok = !more() || issue_qk(0);
            bool begins = true;
            for (int j = 0; ok && more(); ++j) {
                const bool early = next.step != 0;   // a tile's first product waits for its queries: behind the last product of the tile before it
                if (early && more_qk() && !issue_qk(j + 1)) break;
                const int st = j & 1, u = j >> 1;
                if (!mbar_wait(p_full(st), (uint32_t)(u & 1), abort_flag, p.wait_status, 46)) break;
                if (!mbar_wait(v_full(st), (uint32_t)(u & 1), abort_flag, p.wait_status, 47)) break;
                tc_fence_after();
                const uint32_t pa = tmem_base + kColS + (uint32_t)st * kPrefixStep;   // two positions per column: first terms, then second ones
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                    for (int ks = 0; ks < kPrefixStep / 16; ++ks)
                        umma_bf16_ts(tmem_base + kColO, pa + (uint32_t)(term * 32 + ks * 8), dv[st] + (uint64_t)(ks * (2048 >> 4)), idesc_pv,
                                     !begins || term != 0 || ks != 0);
                umma_commit(pv_done(st));
                begins = at.step + 1 == at.plan.steps;
                advance(p, at);
                if (!early && more_qk() && !issue_qk(j + 1)) break;
            }
        }
    } else {   // ---------------- softmax: a query row per thread ----------------
        const int quarter = warp & 3, r = quarter * 32 + lane;   // the quarter of tensor memory's lanes that this warp may touch
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16, to = tmem_base + lane_addr + kColO;
        bool ok = true, begins = true;
        long long out_row = -1;                                  // among the results
        bool idle = false;                                       // no query of this warp counts
        float m_used = -INFINITY, l = 0.f;
        auto begin_tile = [&]() {
            const int member = r / p.group, nth = at.tile * p.per_tile + member;
            const bool valid = member < p.per_tile && nth < at.plan.members && takes_prefix(at.plan.prefix, p.lens[at.plan.b0 + nth]);
            out_row = valid ? (long long)at.plan.b0 * p.n_q + ((long long)at.head * at.plan.members + nth) * p.group + (r - member * p.group) + kPrefixRows * cta : -1;
            idle = !__any_sync(0xffffffffu, valid);
        };
        // pages that the pool does not have: a lane's 16 positions of a step, looked up a step ahead
        auto has_page = [&](const Step &x) {
            const int pos = x.step * kPrefixStep + 16 * (lane & 3);
            return pos >= x.plan.prefix || (unsigned)p.c.table[(long long)x.plan.b0 * p.c.pages_per_seq + (pos >> p.c.page_shift)] < (unsigned)p.c.n_pages;
        };
        bool has = true;
        if (more()) {
            has = has_page(at);
            begin_tile();
        }
        for (int j = 0; more(); ++j) {
            const int st = j & 1, u = j >> 1, p0 = at.step * kPrefixStep;
            ok = __all_sync(0xffffffffu, mbar_wait(s_full(st), (uint32_t)(u & 1), abort_flag, p.wait_status, 48));
            if (!ok) break;
            tc_fence_after();
            const uint32_t there = __ballot_sync(0xffffffffu, has) & 0xfu;   // per 16 positions
            Step next = at;
            advance(p, next);
            const bool last = next.index >= t1 || next.g >= p.groups.n_groups, ends = at.step + 1 == at.plan.steps;
            if (!last) has = has_page(next);
            if (idle) {   // (its rows of P are whatever the scores' bits are, and nobody's)
                mbar_arrive(p_full(st));
                at = next;
                if (ends && !last) begin_tile();
                continue;
            }
            const uint32_t ts = tmem_base + lane_addr + kColS + (uint32_t)st * kPrefixStep;
            uint32_t sv[2][32];
            tmem_ld32_nowait(ts, sv[0]);
            tmem_ld32_nowait(ts + 32u, sv[1]);
            tmem_wait_ld();
            if (p.flip) {
#pragma unroll
                for (int e = 0; e < 32; ++e) { sv[0][e] ^= p.flip; sv[1][e] ^= p.flip; }
            }
            if (p0 + kPrefixStep > at.plan.prefix || there != 0xfu) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (p0 + 32 * c + e >= at.plan.prefix || !(there >> (2 * c + e / 16) & 1u)) sv[c][e] = 0xff800000u;   // -infinity
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 32; e += 8)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx[i] = top3(mx[i], __uint_as_float(sv[c][e + 2 * i]), __uint_as_float(sv[c][e + 2 * i + 1]));
            const float m_step = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
            if (begins) {
                m_used = m_step;
            } else {
                // the maximum that O refers to moves only when a step passes it by 2^8
                const bool need = out_row >= 0 && m_step > m_used + kLazyMax;
                if (__any_sync(0xffffffffu, need)) {
                    ok = __all_sync(0xffffffffu, mbar_wait(pv_done((j - 1) & 1), (uint32_t)(((j - 1) >> 1) & 1), abort_flag, p.wait_status, 49));
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
            const float ref = (m_used == -INFINITY ? 0.f : m_used) - kLift;   // nothing attended so far: every weight is 0
            const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), neg = make_float2(-ref, -ref);
            float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t hi[16], lo[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv[c][2 * e]), __uint_as_float(sv[c][2 * e + 1])), scale2, neg);
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
                tmem_st16(ts + 16u * c, hi);
                tmem_st16(ts + 32u + 16u * c, lo);
            }
            l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(p_full(st));
            at = next;
            begins = ends;
            if (!ends && !last) continue;
            // ---- the share's part of a tile is done ----
            const long long row = out_row;
            if (!last) begin_tile();
            ok = __all_sync(0xffffffffu, mbar_wait(pv_done(st), (uint32_t)(u & 1), abort_flag, p.wait_status, 50));
            if (!ok) break;
            tc_fence_after();
            const bool store = row >= 0 && NNC_BC(row < p.part_rows, 3602);
            if (store) p.s.ml[row] = make_float2(m_used == -INFINITY && l == 0.f ? -INFINITY : ref, l);
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t t[32];
                tmem_ld32(to + 32u * c, t);
                if (!store) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) store16(p.s.o + (8 * c + e) * p.part_rows + row, t + 4 * e);
            }
            tc_fence_before();
            m_used = -INFINITY;
            l = 0.f;
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
// Its query heads' rows are neighbours in every piece.  A thread takes four elements of a row, of every kth piece where rows are few; the
// weights of up to kJoinPieces pieces are computed first, by a warp a row.

constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 8;           // query heads at a time
constexpr int kJoinPieces = kPrefixMaxCtas;

struct JoinParams {
    PagedView c;
    PrefixGroups groups;
    PrefixScratch s;
    const int32_t *lens;
    char *out;
    float *lse;
    long long out_stride, part_rows;
    int group, per_tile, n_q;
};

template <int D, bool BF>   // BF: results (and the cache) are bf16, otherwise fp16
__global__ void __launch_bounds__(kJoinThreads) attn_prefix_join_kernel(const JoinParams p) {
    constexpr int kPieces4 = D / 4;                                // of a row
    __shared__ float wgt[kJoinRows][kJoinPieces + 1];              // of every piece, then of the tail
    __shared__ float2 tot[kJoinRows];                              // reference, sum
    __shared__ float4 sums[kJoinThreads];
    __shared__ uint32_t odd_bits[D];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.x / p.c.n_kv, head = blockIdx.x - b * p.c.n_kv;
    const int g = group_of(p.groups, b);
    long long first_row = 0;
    int n = 0, b0 = 0, prefix = 0;
    if (g >= 0) {
        const PrefixPlan plan = p.s.plan[g];
        if (plan.steps && takes_prefix(plan.prefix, p.lens[b])) {
            b0 = plan.b0;
            prefix = plan.prefix;
            const long long lo = plan.base + ((long long)head * plan.tiles + (b - b0) / p.per_tile) * (plan.steps + kPrefixFixed), share = p.s.head->share;
            const long long c_lo = lo / share;
            n = (int)((lo + plan.steps - 1) / share - c_lo) + 1;
            first_row = (long long)b0 * p.n_q + ((long long)head * plan.members + b - b0) * p.group + kPrefixRows * c_lo;
            if (!NNC_BC(first_row >= 0 && n <= kJoinPieces && first_row + (long long)kPrefixRows * (n - 1) + p.group <= p.part_rows, 3603)) n = 0;
        }
    }
    for (int h0 = 0; h0 < p.group; h0 += kJoinRows) {
        const int rows = min(kJoinRows, p.group - h0);
        const long long q_row = (long long)b * p.n_q + (long long)head * p.group + h0;
        if (warp < rows) {
            const float tail = p.s.tail_lse[q_row + warp] * 1.4426950408889634f;   // the tail's sum is 1 at this reference
            float top = tail;
            for (int i = lane; i < n; i += 32) top = fmaxf(top, p.s.ml[first_row + h0 + warp + (long long)kPrefixRows * i].x);
            top = warp_max(top);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            for (int i = lane; i < n; i += 32) {
                const float2 ml = p.s.ml[first_row + h0 + warp + (long long)kPrefixRows * i];
                const float w = exp2f(ml.x - ref);
                wgt[warp][i] = w;
                sum = fmaf(w, ml.y, sum);
            }
            sum = warp_sum(sum);
            const float w = exp2f(tail - ref);
            if (lane == 0) {
                wgt[warp][n] = w;
                tot[warp] = make_float2(ref, sum + w);
                if (p.lse) p.lse[q_row + warp] = sum + w == 0.f ? -INFINITY : (ref + log2f(sum + w)) * kLn2;
            }
        }
        __syncthreads();
        // thread: element group c4 of row h, pieces k, k + apart, ..
        const int items = rows * kPieces4, apart = kJoinThreads / items;
        {
            const int item = tid % items, k = tid / items;
            const bool mine = k < apart;
            const int h = mine ? item % rows : 0, c4 = mine ? item / rows : 0;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mine) {
                const float4 *src = p.s.o + c4 * p.part_rows + first_row + h0 + h;
#pragma unroll 8
                for (int i = k; i < n; i += apart) {
                    const float w = wgt[h][i];
                    const float4 v = src[(long long)kPrefixRows * i];
                    sum.x = fmaf(w, v.x, sum.x); sum.y = fmaf(w, v.y, sum.y); sum.z = fmaf(w, v.z, sum.z); sum.w = fmaf(w, v.w, sum.w);
                }
                if (k == 0) {
                    const float w = wgt[h][n];
                    const float4 v = *reinterpret_cast<const float4 *>(p.s.tail + (q_row + h) * D + 4 * c4);
                    sum.x = fmaf(w, v.x, sum.x); sum.y = fmaf(w, v.y, sum.y); sum.z = fmaf(w, v.z, sum.z); sum.w = fmaf(w, v.w, sum.w);
                }
            }
            if (apart > 1) {
                sums[tid] = sum;
                __syncthreads();
                if (mine && k == 0)
                    for (int j = 1; j < apart; ++j) {
                        const float4 v = sums[item + j * items];
                        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                    }
            }
            const bool store = mine && k == 0;
            // A column of values with an infinity in an attended row is that infinity, however small the row's weight (two of different signs,
            // or NaN, leave no number); a weight of 0 made NaN of it.  So where a sum is no number the rows are looked through again.
            if (__syncthreads_or(store && !(fabsf((sum.x + sum.y) + (sum.z + sum.w)) < INFINITY))) {
                if (tid < D) {
                    uint32_t bits = 0;
                    const int end = n > 0 ? prefix : 0;
#pragma unroll 4
                    for (int pos = 0; pos < end; ++pos) {
                        const int page = p.c.table[(long long)b0 * p.c.pages_per_seq + (pos >> p.c.page_shift)];
                        if ((unsigned)page >= (unsigned)p.c.n_pages) continue;
                        constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
                        const uint32_t x = reinterpret_cast<const uint16_t *>(p.c.v)[paged_row(p.c, page, head, pos & ((1 << p.c.page_shift) - 1)) * D + tid], size = x & 0x7fffu;
                        if (size >= kInf) bits |= size > kInf ? 4u : x == size ? 1u : 2u;
                    }
                    odd_bits[tid] = bits;
                }
                __syncthreads();
                if (store) {
                    float *const s[4] = {&sum.x, &sum.y, &sum.z, &sum.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t bits = odd_bits[4 * c4 + e];
                        const float behind = p.s.tail[(q_row + h) * D + 4 * c4 + e];
                        if (!(fabsf(behind) < INFINITY)) bits |= behind != behind ? 4u : behind > 0.f ? 1u : 2u;
                        if (bits) *s[e] = bits == 1u ? INFINITY : bits == 2u ? -INFINITY : __uint_as_float(0x7fffffffu);
                    }
                }
            }
            if (store) {
                const float L = tot[h].y, inv = L == 0.f ? 0.f : 1.f / L;
                const long long at = b * p.out_stride + ((long long)head * p.group + h0 + h) * D + 4 * c4;
                uint2 v;
                if constexpr (BF) v = make_uint2(round_bf16x2(sum.x * inv, sum.y * inv), round_bf16x2(sum.z * inv, sum.w * inv));
                else {
                    const __half2 lo = __floats2half2_rn(sum.x * inv, sum.y * inv), hi = __floats2half2_rn(sum.z * inv, sum.w * inv);
                    v = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
                }
                *reinterpret_cast<uint2 *>(p.out + at * 2) = v;
            }
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
    s.head = (PrefixHead *)take(sizeof(PrefixHead));
    s.plan = (PrefixPlan *)take(sizeof(PrefixPlan) * batch);
    s.ml = (float2 *)take(8 * part_rows);
    s.o = (float4 *)take(4 * part_rows * d);
    s.tail_lse = (float *)take(4ll * batch * n_q);
    s.tail = (float *)take(4ll * batch * n_q * d);
    if (bytes) *bytes = used;
    return s;
}
long long part_rows_of(int batch, int n_q) { return (long long)batch * n_q + (long long)kPrefixRows * kPrefixMaxCtas; }

// the pool of one kind as rows of a KV head's positions
bool make_pool_map(CUtensorMap *map, const nnc_paged_kv &c, const void *pool, int box) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.n_pages * c.n_kv_heads * c.page_size}, strides[1] = {(cuuint64_t)c.head_dim * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, one[2] = {1, 1};
    return enc(map, c.type == NNC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(pool), dims, strides, boxes, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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

template <int D, bool BF> cudaError_t launch_prefix_of(const LaunchCtx &lc, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PrefixParams &p) {
    static unsigned long long raised = 0;
    auto kern = attn_prefix_kernel<D, BF>;
    if (cudaError_t e = ensure_dynamic_smem(kern, Tiles<D>::kSmem, &raised); e != cudaSuccess) return e;
    const int ctas = 2 * lc.sm_count < kPrefixMaxCtas ? 2 * lc.sm_count : kPrefixMaxCtas;
    return launch_smem(lc, kern, dim3((unsigned)ctas), dim3(kThreads), (size_t)Tiles<D>::kSmem, mq, mk, mv, p);
}

template <int D> cudaError_t launch_join_of(const LaunchCtx &lc, const JoinParams &p, bool bf, long long ctas) {
    return bf ? launch(lc, attn_prefix_join_kernel<D, true>, dim3((unsigned)ctas), dim3(kJoinThreads), p)
              : launch(lc, attn_prefix_join_kernel<D, false>, dim3((unsigned)ctas), dim3(kJoinThreads), p);
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
    // Every sequence's own rows, the shared ones among them: fp32 and codes; more query heads than a tile has rows, which share rows among
    // themselves; queries whose rows overlap, which a tensor map does not describe.
    if (type == NNC_F32 || cache.type == NNC_E4M3 || n_q_heads / cache.n_kv_heads > kPrefixRows || (batch > 1 && q_stride < (int64_t)n_q_heads * cache.head_dim))
        return launch_attn_paged(lc, q, cache, lens, out, lse, type, batch, n_q_heads, q_stride, out_stride, scale, 0, scratch, NNC_ATTN_PAGED_SCRATCH_BYTES);
    const int d = cache.head_dim, group = n_q_heads / cache.n_kv_heads;
    const bool bf = cache.type == NNC_BF16;
    const PrefixScratch s = carve((char *)scratch + NNC_ATTN_PAGED_SCRATCH_BYTES, batch, n_q_heads, d, part_rows_of(batch, n_q_heads), nullptr);
    const PrefixGroups groups{starts, shared, n_groups, batch};
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
    cudaError_t e = d == 64 ? (bf ? launch_prefix_of<64, true>(early, mq, mk, mv, p) : launch_prefix_of<64, false>(early, mq, mk, mv, p))
                            : (bf ? launch_prefix_of<128, true>(early, mq, mk, mv, p) : launch_prefix_of<128, false>(early, mq, mk, mv, p));
    if (e != cudaSuccess) return e;
    e = launch_attn_tail(lc, q, cache, lens, groups, s.tail, s.tail_lse, type, n_q_heads, q_stride, scale, scratch, NNC_ATTN_PAGED_SCRATCH_BYTES);
    if (e != cudaSuccess) return e;
    JoinParams j = {};
    j.c = p.c; j.groups = groups; j.s = s; j.lens = lens;
    j.out = (char *)out; j.lse = lse; j.out_stride = out_stride; j.part_rows = p.part_rows; j.group = group; j.per_tile = p.per_tile; j.n_q = n_q_heads;
    const long long ctas = (long long)batch * cache.n_kv_heads;
    return d == 64 ? launch_join_of<64>(early, j, bf, ctas) : launch_join_of<128>(early, j, bf, ctas);
}

}  // namespace nnc
