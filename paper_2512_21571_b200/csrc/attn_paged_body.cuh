// Attention of one new token per sequence over a paged key-value cache, sequences of any lengths.  What a (sequence, KV head) attends to
// is a type (`W`) that each operation defines in its own file: whole sequences (attn_paged.cu), what lies behind a shared prefix
// (attn_prefix_tail.cu), listed pages (attn_selected.cu).
//
//   s_n = scale q.k_n,  o = sum_n exp(s_n - m) v_n / sum_n exp(s_n - m),  n over the attended positions
//
// Bound by reading every attended key and value row once.  How it gets there:
//   - The work is a list of tiles (4 warps' blocks of positions of one sequence and KV head; its query heads ride along in
//     groups of up to 16), in the order sequence, head, position, with one more place per head for what it costs to begin and
//     to end it.  The lengths live on the device, so every CTA adds up the list itself and takes an equal contiguous share.
//     A share may end inside a (sequence, head): such pieces leave partial results (m, l, o~) that the CTA finishing last joins in
//     list order (a ticket word; nobody waits), so the result does not depend on who was last.
//   - A warp owns 4 KB of key rows and as much of value rows of every tile and runs its own ring of shared-memory stages, filled by
//     16-byte asynchronous copies that run ahead across heads and sequences; no barrier in the steady state.  Rows outside the
//     attended range are filled with zeros instead of being read, so nothing stored there can reach a product.
//   - Two or three CTAs per SM: three (168 registers, rings of two stages, up to 20 bytes spilled) where that is faster.  32 x 8192, codes,
//     4 query heads of 128 elements per KV head: 114.6 us with two, 99.1 with three; 16 heads of 64: bf16 128.7 and 115.4, but codes
//     98.0 and 100.7 (48 bytes spilled); two operands of 128 elements need 255 registers as it is.
//   - Both products run on the warp-level tensor-core path in transposed form: S^T = K Q^T and O^T = V^T P^T, so 16
//     positions (16 head-dimension elements) fill the 16-row operand and 8 query heads are the 8-column operand: the tensor pipe is
//     busy 17 % of the time at 94 % of the measured copy bandwidth.  A tcgen05 tile would have 128 rows for the same 8 columns,
//     for more of a pipe that does not limit.
//   - E4M3 codes are fp16 values exactly; key scales multiply the scores, value scales (powers of two) are added to the
//     exponents of the probabilities that weigh the codes, so no code is ever multiplied by a scale.  Those weights have a running
//     maximum of their own, over the rows that are not all zeros: the softmax's sum is taken of the probabilities themselves, whose reach
//     has nothing to do with the values'.  (Looking for rows of zeros: 32 x 8192 with heads of 128 97.3 -> 99.1 us, of 64 63.0 -> 67.4.  The
//     warp-level product of 8-bit operands took longer than these conversions and fp16 products: 147 -> 179 us on a ragged batch.)
// Numerics: scores, maxima, sums and outputs are fp32.  Queries enter exactly (16-bit types) or as three bf16 or two fp16 terms, and
// probabilities as three bf16 or two fp16 terms whatever the results' type: 24 and 22 bits, so that the only rounding a caller
// sees is the result's.  (One term less for 16-bit results moved them by up to 2^-18, bf16 results of codes by 2^-12, and took, 32 x 8192 with 4 and 16
// query heads per KV head: bf16 174 and 173 us instead of 174 and 188, codes 98 and 143 instead of 102 and 157.)
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "paged.cuh"

namespace nnc {

namespace {

constexpr int kWarps = 4;
constexpr float kLn2 = 0.69314718055994530942f;
// partial results that one CTA joins: up to Shape::kMaxJoin at once, in groups of kJoinGroup first where there are more (one SM reads
// them at some 100 GB/s, so a long list is cheaper in two rounds)
constexpr int kJoinGroup = 16;

struct PagedAttnParams {
    PagedView c;
    const char *q;
    char *out;
    float *lse;   // where W::kSums, a pair of floats each: the weights' reference (log2 units) and their sum
    const int32_t *lens;
    float *part;
    uint32_t *tickets;
    size_t part_floats;
    long long q_stride, out_stride;   // elements
    int batch, group, chunks, window;   // chunks: groups of NT * 8 query heads per KV head, one row of the grid each
    float scale_log2;
    const int32_t *list, *counts;    // listed pages of every (sequence, KV head): [list_len], how many count
    int list_len;
    const int32_t *starts, *shared;  // groups of sequences: the first of each and the end; positions that they share
    int n_groups, least;
};

template <int D, int NT, int KV, int TYPE>
struct Shape {
    static constexpr int kCtas = (NT == 1 && (TYPE != NNC_F32 || KV != NNC_BF16)) || (NT == 2 && D == 64 && TYPE != NNC_F32 && KV != NNC_E4M3) ? 3 : 2;   // resident per SM
    static constexpr int kBytes = KV == NNC_E4M3 ? 1 : 2;
    static constexpr int kRow = D * kBytes;                  // bytes of a row
    static constexpr int kPB = 4096 / kRow;                  // positions of a warp's block: 4 KB of keys, as many of values
    static constexpr int kSub = kPB / 16;
    static constexpr int kTile = kWarps * kPB;
    static constexpr int kData = 2 * kPB * kRow;             // K rows, then V rows
    static constexpr int kStage = kData + (KV == NNC_E4M3 ? 2 * kPB : 0);   // then K scales, V scales
    static constexpr int kStages = kCtas == 3 ? 2 : 3;
    static constexpr int kTilesD = D / 16;                   // 16-row tiles of O^T
    static constexpr int kOwn = kTilesD / kWarps;            // tiles that a warp merges
    static constexpr int kRounds = kCtas == 3 ? kOwn : 1;    // warps hand their tiles to one another in so many rounds,
    static constexpr int kOnce = kOwn / kRounds;             // so many tiles a warp at once,
    static constexpr int kHand = kWarps * 3 * kOnce * 4 * 32 * 4;   // in so many bytes,
    static constexpr int kMaxJoin = NT == 1 ? 64 : 32;
    static constexpr int kJoin = 8 * NT * kMaxJoin * 12 + 8 * NT * 8;   // or (m, l), weights and sums where results are joined
    static constexpr int kComb = kHand > kJoin ? kHand : kJoin;
    static constexpr int kSmem = kWarps * kStages * kStage + kComb;
    static constexpr int kSlotFloats = 8 * NT * (D + 2);     // a partial result: o~ of 8 NT heads, then their (m, l)
};

struct AttnShared {
    float ml[kWarps][8][3];   // references of o~ and of l, and l
    int sums[kWarps];
    uint32_t odd[32];   // what a piece's values hold besides finite numbers (odd_values)
    int first_b, first_head, first_rest;
    struct { int c_lo, c_hi, q_head, heads_here, b, last; } split[2];   // this CTA's partial results: slot 0's and slot 1's
};

// byte offset of 16-byte piece c of row r, arranged so that eight rows of one column of pieces lie in different banks
template <int ROW> __device__ __forceinline__ int swizzled(int r, int c) {
    if constexpr (ROW >= 128) return r * ROW + ((c ^ (r & 7)) << 4);
    else return (r >> 1) * 128 + ((((r & 1) << 2 | c) ^ ((r >> 1) & 7)) << 4);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_or_zeros(uint32_t dst, const void *src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <bool BF>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]) {
    if constexpr (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}

// transposes an 8x8 matrix of 16-bit elements held one row per 4 lanes
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// 2^x; what is below 2^-126 is 0
__device__ __forceinline__ float exp2_flush(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// four E4M3 codes as two fp16 pairs: the low two, the high two
__device__ __forceinline__ void codes_to_f16(uint32_t codes, uint32_t &lo, uint32_t &hi) {
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(lo), "=r"(hi) : "r"(codes));
}

// x, y as sums of N terms of 16 bits (each term the rounding of what the ones before it leave)
template <bool BF, int N> __device__ __forceinline__ void split(float x, float y, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (BF) {
            t[i] = pack_bf16x2(x, y);
            if (i + 1 < N) { x -= bf16_lo(t[i]); y -= bf16_hi(t[i]); }
        } else {
            const __half2 h = __floats2half2_rn(x, y);
            t[i] = *reinterpret_cast<const uint32_t *>(&h);
            if (i + 1 < N) { x -= __low2float(h); y -= __high2float(h); }
        }
    }
}

// What a (sequence, KV head) attends to: positions [start, end), and its tiles, counted from `start` rounded down to 16.  Where pages
// are listed, positions are counted through the list, and `len` says which of them the sequence has.
struct Reach {
    int start, end, tiles, len;
    // places of a (sequence, head) in the list: its tiles and one for what it costs to begin and to end
    __device__ __forceinline__ int places() const { return tiles ? tiles + 1 : 0; }
};
__device__ __forceinline__ int length_of(const PagedAttnParams &p, int len) { return max(0, min(len, p.c.pages_per_seq << p.c.page_shift)); }
template <int TILE> __device__ __forceinline__ Reach reach_between(int start, int end) {
    return Reach{start, end, (end - (start & ~15) + TILE - 1) / TILE, end};
}
constexpr int kNoPage = -1, kNoRows = -2;   // instead of a page: an entry that the pool does not have; positions that the sequence does not

// a tile, and its place in the list
struct Place {
    Reach r;
    int b, head, tile;   // head: KV head
    int index;
};
template <int TILE, typename W> __device__ __forceinline__ void step(const PagedAttnParams &p, Place &at) {
    ++at.index;
    if (++at.tile < at.r.tiles) return;
    ++at.index;
    at.tile = 0;
    ++at.head;
    if constexpr (W::kListed) {
        do {
            if (at.head >= p.c.n_kv) { at.head = 0; ++at.b; }
            if (at.b >= p.batch) { at.r = Reach{0, 0, 0, 0}; return; }   // past the list's end: nothing is taken from here
            at.r = W::template reach<TILE>(p, at.b, at.head);
            if (at.r.tiles == 0) ++at.head;
        } while (at.r.tiles == 0);
    } else {
        if (at.head < p.c.n_kv) return;
        at.head = 0;
        do {
            if (++at.b >= p.batch) { at.r = Reach{0, 0, 0, 0}; return; }
            at.r = W::template reach<TILE>(p, at.b, 0);
        } while (at.r.tiles == 0);
    }
}

// Counts a CTA that has written its piece, after a barrier of its threads; true for the last of n, which leaves the word at
// zero.  Release and acquire of this one thread, with the barriers around it, order the CTA's stores and loads.
__device__ __forceinline__ bool take_ticket(uint32_t *ticket, int n) {
    uint32_t before;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(ticket) : "memory");
    if (before != (uint32_t)(n - 1)) return false;
    *ticket = 0u;
    return true;
}

template <int TYPE> __device__ __forceinline__ void store_out(const PagedAttnParams &p, long long at, float v) {
    if constexpr (TYPE == NNC_F32) reinterpret_cast<float *>(p.out)[at] = v;
    else if constexpr (TYPE == NNC_BF16) reinterpret_cast<uint16_t *>(p.out)[at] = f32_to_bf16_bits(v);
    else reinterpret_cast<__half *>(p.out)[at] = __float2half_rn(v);
}

// NT: groups of 8 query heads; TYPE: the queries' and the results'.  W::kSums: results are the sums in 32 bits, not divided by the weights' sum, which
// goes out beside them
template <int D, int NT, int KV, int TYPE, typename W>
__device__ __forceinline__ void attn_paged_cta(const PagedAttnParams &p) {
    typedef Shape<D, NT, KV, TYPE> S;
    constexpr bool BF = KV == NNC_BF16, CODES = KV == NNC_E4M3;
    constexpr int OUT = W::kSums ? NNC_F32 : TYPE;
    constexpr int PT = BF ? 3 : 2, QT = TYPE == NNC_F32 ? PT : 1;   // terms of the probabilities and of the queries
    constexpr int PB = S::kPB, TILE = S::kTile, ROW = S::kRow;
    // fp16 probabilities are scaled by 2^14, so that small ones keep their bits (the sums are scaled alike)
    constexpr float kLift = BF ? 0.f : 14.f;
    extern __shared__ __align__(128) char smem[];
    __shared__ AttnShared sh;
    pdl_launch_dependents();
    if constexpr (!W::kConcurrent) pdl_wait();   // lengths, tables, queries and rows may be the preceding kernel's
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // the same in all lanes, which the compiler then knows
    const int g8 = lane >> 2, t4 = lane & 3;
    // ---- the list: how many places there are, and where this CTA's share begins ----
    const int heads = W::kListed ? 1 : p.c.n_kv, most = p.c.pages_per_seq << p.c.page_shift;   // heads: that a sum over a sequence stands for
    const int per = (p.batch + kWarps * 32 - 1) / (kWarps * 32);
    const int b_lo = min(tid * per, p.batch), b_hi = min(b_lo + per, p.batch);
    int mine = 0, odd = 0;   // odd: an empty sequence, or a length that does not fit
    for (int b = b_lo; b < b_hi; ++b) {
        const int len = p.lens[b];
        odd |= len <= 0 || len > most;
        if constexpr (W::kListed) {
            for (int h = 0; h < p.c.n_kv; ++h) {
                const int n = W::template reach<TILE>(p, b, h).places();
                odd |= n == 0;
                mine += n;
            }
        } else {
            const int n = W::template reach<TILE>(p, b, 0).places();
            odd |= n == 0;
            mine += n;
        }
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sh.sums[warp] = incl;
    auto store_weights = [&](long long at, float m, float l) {
        if constexpr (W::kSums) reinterpret_cast<float2 *>(p.lse)[at] = make_float2(m, l);
        else p.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    };
    auto inverse = [](float l) { return W::kSums ? 1.f : l == 0.f ? 0.f : 1.f / l; };
    if (__syncthreads_or(odd)) {   // zeros for sequences with nothing to attend to; lengths that do not fit are reported
        for (int b = blockIdx.y == 0 ? blockIdx.x : p.batch; b < p.batch; b += gridDim.x) {
            const int n_q = p.c.n_kv * p.group;
            if (p.lens[b] > most && tid == 0) paged_complain(p.c);
            for (int h = 0; h < (W::kListed ? p.c.n_kv : 1); ++h) {
                if (W::template reach<TILE>(p, b, h).tiles > 0) continue;
                const int first = h * p.group, end = W::kListed ? first + p.group : n_q;   // query heads
                for (int i = first * D + tid; i < end * D; i += kWarps * 32) store_out<OUT>(p, b * p.out_stride + i, 0.f);
                if (p.lse) for (int i = first + tid; i < end; i += kWarps * 32) store_weights((long long)b * n_q + i, -INFINITY, 0.f);
            }
        }
    }
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { if (w < warp) before += sh.sums[w]; all += sh.sums[w]; }
    const int total = all * heads;                             // places; the host bounds them by 2^30
    const int share = (total + gridDim.x - 1) / gridDim.x;     // of every CTA but the last ones
    const int cta = blockIdx.x, chunk = blockIdx.y;            // chunk: which 8 NT query heads of every KV head
    float *const part = p.part + (size_t)chunk * gridDim.x * 2 * S::kSlotFloats;
    uint32_t *const tickets = p.tickets + chunk * gridDim.x;
    if ((long long)cta * share >= total) return;
    const int t0 = cta * share, t1 = min(t0 + share, total);
    {
        const int lo = (before + incl - mine) * heads;
        if (t0 >= lo && t0 - lo < mine * heads) {
            int rest = t0 - lo, b = b_lo, h = 0;
            for (; b < b_hi; W::kListed && h + 1 < p.c.n_kv ? ++h : (h = 0, ++b)) {
                const int n = W::template reach<TILE>(p, b, h).places() * heads;
                if (rest < n) break;
                rest -= n;
            }
            sh.first_b = b;
            sh.first_head = h;
            sh.first_rest = rest;
        }
    }
    if (tid < 2) sh.split[tid].c_lo = -1;
    __syncthreads();
    Place ahead;   // where the copies are
    ahead.b = sh.first_b;
    ahead.r = W::template reach<TILE>(p, ahead.b, sh.first_head);
    if constexpr (W::kListed) {
        ahead.head = sh.first_head;
        ahead.tile = sh.first_rest;
    } else {
        ahead.head = sh.first_rest / ahead.r.places();
        ahead.tile = sh.first_rest - ahead.head * ahead.r.places();
    }
    ahead.index = t0;
    if (ahead.tile == ahead.r.tiles) { --ahead.index; --ahead.tile; step<TILE, W>(p, ahead); }   // the place after its tiles
    if (ahead.index >= t1) return;
    Place now = ahead;   // where the products are

    // ---- copies of this warp's block of a tile ----
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S::kStages * S::kStage);
    int pages[S::kSub], held[S::kSub];   // held: listed pages: how many of the 16 positions the sequence has
    auto find_pages = [&]() {   // one step before they are needed
        const int p0 = (ahead.r.start & ~15) + ahead.tile * TILE + warp * PB;
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
            pages[u] = kNoPage;
            if (p0 + 16 * u < ahead.r.end) pages[u] = W::page(p, ahead, p0 + 16 * u, held[u]);
        }
    };
    // per 16 positions of each stage: a bit, its page exists; where pages are listed five, how many of its rows count
    constexpr int kHeldBits = W::kListed ? 5 : 1;
    constexpr uint32_t kHeldMask = (1u << (kHeldBits * S::kSub)) - 1u;
    typename std::conditional<W::kListed, unsigned long long, uint32_t>::type present = 0;
    constexpr int kPieces = ROW / 16, kRowsPerStep = 32 / kPieces, kSteps = 16 / kRowsPerStep;
    const int r0 = lane / kPieces, c0 = lane % kPieces;   // this lane's row and piece in the first step of 16 rows
    auto request = [&](int stage) {
        const int p0 = (ahead.r.start & ~15) + ahead.tile * TILE + warp * PB;
        const uint32_t base = ring + stage * S::kStage;
        present &= ~((decltype(present))kHeldMask << (stage * S::kSub * kHeldBits));
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
            const int pb = p0 + 16 * u;
            if (pb >= ahead.r.end) break;
            const bool there = (unsigned)pages[u] < (unsigned)p.c.n_pages && NNC_BC(ahead.b < p.batch && ahead.head < p.c.n_kv && stage < S::kStages, 3202);
            const bool all = W::kListed ? held[u] == 16 : pb >= ahead.r.start && pb + 16 <= ahead.r.end;
            const long long row = there ? paged_row(p.c, pages[u], ahead.head, pb & ((1 << p.c.page_shift) - 1)) : 0;
            if (!NNC_BC(row >= 0 && row + 16 <= paged_rows(p.c), 3203)) continue;
            const char *ks = p.c.k + row * ROW + lane * 16, *vs = p.c.v + row * ROW + lane * 16;   // 16 rows are one run of bytes
            if (there && all) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const uint32_t dst = base + swizzled<ROW>(16 * u + r0 + i * kRowsPerStep, c0);
                    copy16(dst, ks + i * 512);
                    copy16(dst + PB * ROW, vs + i * 512);
                }
            } else {
                // (a table may hold kNoRows, too: where the sequence has rows that is a page that the pool does not have)
                if (!there && (!W::kListed || pages[u] != kNoRows || held[u] > 0) && lane == 0) paged_complain(p.c);
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const int r = r0 + i * kRowsPerStep;
                    const bool live = there && (W::kListed ? r < held[u] : pb + r >= ahead.r.start && pb + r < ahead.r.end);
                    const uint32_t dst = base + swizzled<ROW>(16 * u + r, c0);
                    copy16_or_zeros(dst, live ? ks + i * 512 : p.c.k, live);
                    copy16_or_zeros(dst + PB * ROW, live ? vs + i * 512 : p.c.v, live);
                }
            }
            if (there) present |= (decltype(present))(W::kListed ? held[u] : 1) << ((stage * S::kSub + u) * kHeldBits);
            if constexpr (CODES) {
                if (lane < 2)
                    copy16_or_zeros(base + S::kData + lane * PB + 16 * u, there ? (lane ? p.c.v_scale : p.c.k_scale) + row : p.c.k_scale, there);
            }
        }
    };

    // ---- per (sequence, head) state ----
    uint32_t qf[NT][QT][D / 16][2];
    float qmul[NT][2];
    float o[NT][S::kTilesD][4], m_run[NT][2], l_run[NT][2];
    float mv_run[NT][2];   // codes: the maximum of score + value exponent, which o~ refers to; otherwise that is m_run
    int piece_first = now.index;   // place of the piece's first tile

    // Queries of a (sequence, head): lane (g8, t4) holds head g8's elements of contraction columns 2 t4, 2 t4 + 1, 2 t4 + 8,
    // 2 t4 + 9 of every step of 16; with codes, a key's four neighbouring codes 4 t4 .. 4 t4 + 3 stand in those columns.
    // They are all requested before any is used, and wait as they are in the fragments' registers.
    auto load_queries = [&](const Place &at_piece) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int g = chunk * (8 * NT) + nt * 8 + g8;
            const long long at = at_piece.b * p.q_stride + (long long)(at_piece.head * p.group + (g < p.group ? g : 0)) * D + (CODES ? 4 : 2) * t4;
            constexpr int kApart = CODES ? 2 : 8;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                if constexpr (TYPE == NNC_F32) {
                    const float *src = reinterpret_cast<const float *>(p.q) + at + 16 * s;
                    const uint2 a = *reinterpret_cast<const uint2 *>(src), b = *reinterpret_cast<const uint2 *>(src + kApart);
                    qf[nt][0][s][0] = a.x; qf[nt][0][s][1] = a.y; qf[nt][QT - 1][s][0] = b.x; qf[nt][QT - 1][s][1] = b.y;
                } else {
                    const uint16_t *src = reinterpret_cast<const uint16_t *>(p.q) + at + 16 * s;
                    qf[nt][0][s][0] = *reinterpret_cast<const uint32_t *>(src);
                    qf[nt][0][s][1] = *reinterpret_cast<const uint32_t *>(src + kApart);
                }
            }
        }
    };
    auto begin_piece = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool there = chunk * (8 * NT) + nt * 8 + g8 < p.group;
            float f[D / 16][4];
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if constexpr (TYPE == NNC_F32) {
                        f[s][e] = __uint_as_float(qf[nt][0][s][e]);
                        f[s][2 + e] = __uint_as_float(qf[nt][QT - 1][s][e]);
                    } else if constexpr (TYPE == NNC_BF16) {
                        f[s][2 * e] = bf16_lo(qf[nt][0][s][e]);
                        f[s][2 * e + 1] = bf16_hi(qf[nt][0][s][e]);
                    } else {
                        const __half2 h = *reinterpret_cast<const __half2 *>(&qf[nt][0][s][e]);
                        f[s][2 * e] = __low2float(h);
                        f[s][2 * e + 1] = __high2float(h);
                    }
                }
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) { if (!there) f[s][e] = 0.f; top = fmaxf(top, fabsf(f[s][e])); }
            float undo = 1.f;
            if constexpr (!BF) {
                // fp16 operands: the row times the power of two that brings its largest magnitude into [2^14, 2^15)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int e8 = (int)(__float_as_uint(top) >> 23);
                const int sh8 = (top == 0.f || e8 >= 255) ? 127 : min(268 - e8, 253);
                const float up = __uint_as_float((uint32_t)sh8 << 23);
                undo = __uint_as_float((uint32_t)(254 - sh8) << 23);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[s][e] *= up;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                qmul[nt][e] = p.scale_log2 * __shfl_sync(0xffffffffu, undo, (2 * t4 + e) * 4);
                m_run[nt][e] = mv_run[nt][e] = -INFINITY;
                l_run[nt][e] = 0.f;
            }
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                uint32_t a[QT], b[QT];
                split<BF, QT>(f[s][0], f[s][1], a);
                split<BF, QT>(f[s][2], f[s][3], b);
#pragma unroll
                for (int i = 0; i < QT; ++i) { qf[nt][i][s][0] = a[i]; qf[nt][i][s][1] = b[i]; }
            }
#pragma unroll
            for (int i = 0; i < S::kTilesD; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
        }
    };

    // asks L2 for the queries of the (sequence, head) that the copies have reached
    auto prefetch_queries = [&]() {
        constexpr int size = TYPE == NNC_F32 ? 4 : 2;
        const int at = (warp * 32 + lane) * 128;   // a line each
        const int q_head = ahead.head * p.group + chunk * (8 * NT), heads_here = min(8 * NT, p.group - chunk * (8 * NT));
        if (at < heads_here * D * size)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.q + (ahead.b * p.q_stride + (long long)q_head * D) * size + at));
    };

    // lane's row and piece in the four 8x8 matrices of an ldmatrix: K (rows = positions) and V (transposed)
    const int lr = lane & 7, lm = lane >> 3;
    auto products = [&](int stage) {
        const int p0 = (now.r.start & ~15) + now.tile * TILE + warp * PB;
        if (p0 >= now.r.end) return;
        const uint32_t kb = ring + stage * S::kStage, vb = kb + PB * ROW;
        const char *scales = smem + warp * (S::kStages * S::kStage) + stage * S::kStage + S::kData;
        // scores.  Even and odd steps (and the lower terms of fp32 queries) have sums of their own: shorter chains, and the tensor
        // cores cut what they add, so shorter chains of large partial sums are nearer to fp32 as well
        float s[S::kSub][NT][4];
        {
            constexpr int kSums = QT > 1 ? 3 : 2;
            float acc[kSums][S::kSub][NT][4];
#pragma unroll
            for (int x = 0; x < kSums; ++x)
#pragma unroll
                for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) acc[x][u][nt][0] = acc[x][u][nt][1] = acc[x][u][nt][2] = acc[x][u][nt][3] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 16; c += 2) {
#pragma unroll
                for (int u = 0; u < S::kSub; ++u) {
                    uint32_t a[2][4];
                    if constexpr (!CODES) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) ldsm4(a[e], kb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, 2 * (c + e) + (lm >> 1)));
                    } else {
                        uint32_t x[4];
                        ldsm4(x, kb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, c + (lm >> 1)));
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            codes_to_f16(x[2 * e], a[e][0], a[e][2]);
                            codes_to_f16(x[2 * e + 1], a[e][1], a[e][3]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < QT; ++i)
                                mma16816<BF>(acc[i == 0 ? e : 2][u][nt], a[e][0], a[e][1], a[e][2], a[e][3], qf[nt][i][c + e]);
                }
            }
#pragma unroll
            for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        s[u][nt][x] = acc[0][u][nt][x] + acc[1][u][nt][x];
                        // (an infinity is the first terms': the lower ones may be 0 or of the other sign, and make NaN of it)
                        if constexpr (QT > 1) s[u][nt][x] += fabsf(s[u][nt][x]) == INFINITY ? 0.f : acc[2][u][nt][x];
                    }
        }
        const uint32_t here = (uint32_t)(present >> (stage * S::kSub * kHeldBits)) & kHeldMask;
        constexpr uint32_t kAll = W::kListed ? 16u * (kHeldMask / 31u) : kHeldMask;
        const bool full = p0 >= now.r.start && p0 + PB <= now.r.end && here == kAll;
        // A row of zeros has no exponent: whatever its scale says, it must not set the maximum for the others.  Two pieces a row tell an
        // ordinary row (are there any bits but signs?); only where some have none there the others are looked at.
        uint32_t filled[S::kSub];   // a bit a row
        if constexpr (CODES) {
            const char *rows = scales - S::kData + PB * ROW;
            auto any_in = [&](int u, int piece) {   // of pieces `piece` and `piece` + 1
                const uint4 x = *reinterpret_cast<const uint4 *>(rows + swizzled<ROW>(16 * u + (lane & 15), piece + (lane >> 4)));
                const uint32_t votes = __ballot_sync(0xffffffffu, ((x.x | x.y | x.z | x.w) & 0x7f7f7f7fu) != 0u);
                return (votes | votes >> 16) & 0xffffu;
            };
            uint32_t all_rows = 0xffffu;
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) all_rows &= filled[u] = any_in(u, 0);
            if (all_rows != 0xffffu) {
#pragma unroll 1
                for (int piece = 2; piece < kPieces; piece += 2)
#pragma unroll
                    for (int u = 0; u < S::kSub; ++u) filled[u] |= any_in(u, piece);
            }
        }
        float ev[S::kSub][2];   // exponents of the value rows
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {   // rows g8 and g8 + 8
                float ks = 1.f;
                if constexpr (CODES) {
                    const uint32_t bk = (uint8_t)scales[16 * u + g8 + 8 * r], bv = (uint8_t)scales[PB + 16 * u + g8 + 8 * r];
                    ks = __uint_as_float(bk << 23);
                    ev[u][r] = __uint_as_float(0x4b000000u | bv) - 8388735.f;   // bv - 127: 2^23 + bv as fp32, no conversion
                    if (!(filled[u] >> (g8 + 8 * r) & 1u)) ev[u][r] = -INFINITY;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float &x = s[u][nt][2 * r + e];
                        x *= CODES ? qmul[nt][e] * ks : qmul[nt][e];
                    }
            }
        }
        if (!full) {
#pragma unroll
            for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int pos = p0 + 16 * u + g8 + 8 * r;
                    if constexpr (W::kListed) {
                        if (g8 + 8 * r < (int)(here >> (5 * u) & 31u)) continue;
                    } else {
                        if ((here >> u & 1u) && pos >= now.r.start && pos < now.r.end) continue;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) s[u][nt][2 * r] = s[u][nt][2 * r + 1] = -INFINITY;
                }
        }
        // ---- online softmax; with codes, a second one of the scores plus the value rows' exponents for what weighs the codes ----
        uint32_t pf[S::kSub][NT][PT][2];
        float alpha[NT][2];
        auto top_of = [&](int nt, int e) {   // of this block's scores
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) mx = fmaxf(mx, fmaxf(s[u][nt][e], s[u][nt][2 + e]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            return fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if constexpr (CODES) {   // a lane's positions have a maximum of their own, until the piece ends
                    float m_new = m_run[nt][e], sum = 0.f;
#pragma unroll
                    for (int u = 0; u < S::kSub; ++u) m_new = fmaxf(m_new, fmaxf(s[u][nt][e], s[u][nt][2 + e]));
                    const float ref = m_new == -INFINITY ? 0.f : m_new;
#pragma unroll
                    for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float &x = s[u][nt][2 * r + e];
                            sum += exp2_flush(x - ref);
                            x += ev[u][r];
                        }
                    l_run[nt][e] = fmaf(l_run[nt][e], exp2_flush(m_run[nt][e] - ref), sum);
                    m_run[nt][e] = m_new;
                }
                float &m = CODES ? mv_run[nt][e] : m_run[nt][e];
                const float m_new = fmaxf(m, top_of(nt, e));
                const float ref = (m_new == -INFINITY ? 0.f : m_new) - kLift;   // nothing attended so far: every weight is 0
                alpha[nt][e] = exp2_flush(m - kLift - ref);
                m = m_new;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float &x = s[u][nt][2 * r + e];
                        x = exp2_flush(x - ref);
                        sum += x;
                    }
                if constexpr (!CODES) l_run[nt][e] = fmaf(l_run[nt][e], alpha[nt][e], sum);
            }
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                uint32_t lo[PT], hi[PT];
                split<BF, PT>(s[u][nt][0], s[u][nt][1], lo);
                split<BF, PT>(s[u][nt][2], s[u][nt][3], hi);
#pragma unroll
                for (int i = 0; i < PT; ++i) { pf[u][nt][i][0] = transpose8(lo[i]); pf[u][nt][i][1] = transpose8(hi[i]); }
            }
        }
        // ---- O^T += V^T P^T.  o[nt][i]: columns are heads 2 t4, 2 t4 + 1; rows are elements 16 i + g8 and 16 i + 8 + g8, or
        //      with codes 16 i + 2 g8 and 16 i + 2 g8 + 1.  A block's products get a sum of their own that is then added in fp32: the
        //      tensor cores cut what they add, always towards zero, which over a share of 131072 positions comes to 2e-4 of the result ----
        int subs = 1;   // 16-position parts that hold anything: what was not copied may be no number
        if constexpr (S::kSub > 1) subs = min(S::kSub, (now.r.end - p0 + 15) >> 4);
#pragma unroll
        for (int i = 0; i < S::kTilesD; i += 2) {
            float fresh[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) fresh[nt][e][0] = fresh[nt][e][1] = fresh[nt][e][2] = fresh[nt][e][3] = 0.f;
#pragma unroll
            for (int u = 0; u < S::kSub; ++u) {
                if (u >= subs) break;
                uint32_t a[2][4];
                if constexpr (!CODES) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) ldsm4_trans(a[e], vb + swizzled<ROW>(16 * u + lr + (lm >> 1) * 8, 2 * (i + e) + (lm & 1)));
                } else {
                    uint32_t x[4];   // positions 0-7 and 8-15 of piece i, then of piece i + 1
                    ldsm4_trans(x, vb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, i + (lm >> 1)));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // a lane holds two neighbouring codes of two positions: pair them by code
                        codes_to_f16(__byte_perm(x[2 * e], 0, 0x3120), a[e][0], a[e][1]);
                        codes_to_f16(__byte_perm(x[2 * e + 1], 0, 0x3120), a[e][2], a[e][3]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < PT; ++j) mma16816<BF>(fresh[nt][e], a[e][0], a[e][1], a[e][2], a[e][3], pf[u][nt][j]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[nt][i + e][x] = fmaf(o[nt][i + e][x], alpha[nt][x & 1], fresh[nt][e][x]);
        }
    };

    // ---- results.  A warp's fragments of O^T tile i: rows d0 (and d1) of two heads ----
    float (*comb)[3][S::kOnce][32][4] = reinterpret_cast<float (*)[3][S::kOnce][32][4]>(smem + kWarps * S::kStages * S::kStage);

    // A column of values with an infinity in an attended row is that infinity, however small the row's weight (two of different signs, or
    // NaN, leave no number).  The products cannot say so: a weight's lower term, or a weight below the smallest, is 0, and 0 or a negative
    // number times infinity makes NaN.  So a piece that ends with anything but finite sums looks through its rows again, a row
    // a warp: three bits a column, for +infinity, -infinity and NaN.
    constexpr int kCols = D / 32;   // columns a lane
    auto odd_values = [&](int p_lo, int p_hi) {
        if (tid < 32) sh.odd[tid] = 0u;
        __syncthreads();
        uint32_t bits = 0;
#pragma unroll 4
        for (int pos = p_lo + warp; pos < p_hi; pos += kWarps) {
            int rows;
            const int page = W::page(p, now, pos & ~15, rows);
            if ((unsigned)page >= (unsigned)p.c.n_pages || (W::kListed && (pos & 15) >= rows)) continue;
            const uint32_t *row = reinterpret_cast<const uint32_t *>(p.c.v + paged_row(p.c, page, now.head, pos & ((1 << p.c.page_shift) - 1)) * ROW) + lane * (kCols / 2);
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
                const uint32_t x = row[i / 2] >> (16 * (i & 1)) & 0xffffu, size = x & 0x7fffu;
                if (size >= kInf) bits |= (size > kInf ? 4u : x == size ? 1u : 2u) << (3 * i);
            }
        }
        if (bits) atomicOr(&sh.odd[lane], bits);
        __syncthreads();
    };
    auto odd_or = [&](int d, float sum) {
        const uint32_t bits = sh.odd[d / kCols] >> (3 * (d % kCols)) & 7u;
        return bits == 0u ? sum : bits == 1u ? INFINITY : bits == 2u ? -INFINITY : __uint_as_float(0x7fffffffu);
    };

    auto end_piece = [&]() {
        const int item_lo = now.index - now.tile, item_hi = item_lo + now.r.tiles;   // places of this (sequence, head)'s tiles
        const int first = piece_first;
        const bool whole = first == item_lo && now.index + 1 == item_hi;
        const int q_head = now.head * p.group + chunk * (8 * NT), heads_here = min(8 * NT, p.group - chunk * (8 * NT));
        const long long out_at = now.b * p.out_stride + (long long)q_head * D, lse_at = (long long)now.b * (p.c.n_kv * p.group) + q_head;
        // partial results: slot 0 of a CTA for a piece that continues an earlier CTA's, slot 1 for one that starts here
        float *slot = part + (size_t)(2 * cta + (first == item_lo ? 1 : 0)) * S::kSlotFloats;
        float all_sums = 0.f;
        if constexpr (!CODES) {   // (a code is never infinite, and NaN comes through by itself)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < S::kTilesD; ++i) all_sums += (o[nt][i][0] + o[nt][i][1]) + (o[nt][i][2] + o[nt][i][3]);
        }
        bool odd = !(fabsf(all_sums) < INFINITY);
        if (!NNC_BC(now.b < p.batch && now.head < p.c.n_kv && heads_here > 0 && (chunk * (8 * NT)) + heads_here <= p.group, 3205)) return;
        if (!whole && !NNC_BC((size_t)(2 * (chunk * gridDim.x + cta) + 2) * S::kSlotFloats <= p.part_floats, 3201)) return;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = l_run[nt][e], m = m_run[nt][e];
                if constexpr (CODES) {
#pragma unroll
                    for (int x = 4; x < 32; x *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                    l *= m_run[nt][e] == -INFINITY ? 1.f : exp2f(m_run[nt][e] - m);   // (no positions: l is 0)
                }
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                if (g8 == 0) {
                    float *const ml = sh.ml[warp][2 * t4 + e];
                    ml[0] = (CODES ? mv_run[nt][e] : m) - kLift;
                    ml[1] = CODES ? m : ml[0];
                    ml[2] = l;
                }
            }
            float M[2], L[2], wgt[kWarps][2];
#pragma unroll
            for (int round = 0; round < S::kRounds; ++round) {
                float own[S::kOnce][4];
#pragma unroll
                for (int to = 0; to < kWarps; ++to)
#pragma unroll
                    for (int j = 0; j < S::kOnce; ++j) {
                        const float (&v)[4] = o[nt][to * S::kOwn + round * S::kOnce + j];
                        if (to == warp) { own[j][0] = v[0]; own[j][1] = v[1]; own[j][2] = v[2]; own[j][3] = v[3]; }
                        else *reinterpret_cast<float4 *>(comb[to][warp < to ? warp : warp - 1][j][lane]) = make_float4(v[0], v[1], v[2], v[3]);
                    }
                if (CODES || nt > 0 || round > 0) __syncthreads();
                else {
                    odd = __syncthreads_or(odd);
                    if (odd) {
                        const int base = now.r.start & ~15;
                        odd_values(max(now.r.start, base + (first - item_lo) * TILE), min(now.r.end, base + (now.tile + 1) * TILE));
                    }
                }
                if (round == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        M[e] = -INFINITY;
#pragma unroll
                        for (int w = 0; w < kWarps; ++w) M[e] = fmaxf(M[e], sh.ml[w][2 * t4 + e][1]);
                        const float ref = M[e] == -INFINITY ? 0.f : M[e];
                        L[e] = 0.f;
#pragma unroll
                        for (int w = 0; w < kWarps; ++w) {
                            const float *const ml = sh.ml[w][2 * t4 + e];
                            wgt[w][e] = exp2f(ml[0] - ref);   // o~ refers to M from here on
                            L[e] = fmaf(CODES ? exp2f(ml[1] - ref) : wgt[w][e], ml[2], L[e]);
                        }
                    }
                }
                float sum[S::kOnce][4];
#pragma unroll
                for (int j = 0; j < S::kOnce; ++j) sum[j][0] = sum[j][1] = sum[j][2] = sum[j][3] = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w)
#pragma unroll
                    for (int j = 0; j < S::kOnce; ++j) {
                        float4 v = make_float4(own[j][0], own[j][1], own[j][2], own[j][3]);
                        if (w != warp) v = *reinterpret_cast<const float4 *>(comb[warp][w < warp ? w : w - 1][j][lane]);
                        sum[j][0] = fmaf(wgt[w][0], v.x, sum[j][0]); sum[j][1] = fmaf(wgt[w][1], v.y, sum[j][1]);
                        sum[j][2] = fmaf(wgt[w][0], v.z, sum[j][2]); sum[j][3] = fmaf(wgt[w][1], v.w, sum[j][3]);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int h = nt * 8 + 2 * t4 + e;
                    if (h >= heads_here) continue;
                    const float inv = inverse(L[e]);
#pragma unroll
                    for (int j = 0; j < S::kOnce; ++j) {
                        const int i = warp * S::kOwn + round * S::kOnce + j;
                        const int d0 = CODES ? 16 * i + 2 * g8 : 16 * i + g8, d1 = CODES ? d0 + 1 : d0 + 8;
                        if (!CODES && odd) { sum[j][e] = odd_or(d0, sum[j][e]); sum[j][2 + e] = odd_or(d1, sum[j][2 + e]); }
                        if (whole) {
                            store_out<OUT>(p, out_at + h * D + d0, sum[j][e] * inv);
                            store_out<OUT>(p, out_at + h * D + d1, sum[j][2 + e] * inv);
                        } else {
                            slot[h * D + d0] = sum[j][e];
                            slot[h * D + d1] = sum[j][2 + e];
                        }
                    }
                    if (round == 0 && warp == 0 && g8 == 0) {
                        if (!whole) *(reinterpret_cast<float2 *>(slot + 8 * NT * D) + h) = make_float2(M[e], L[e]);
                        else if (p.lse) store_weights(lse_at + h, M[e], L[e]);
                    }
                }
                __syncthreads();
            }
        }
        if (!whole && tid == 0) {
            auto &s = sh.split[first == item_lo ? 1 : 0];
            s.c_lo = item_lo / share;          // the CTAs that have a piece of it
            s.c_hi = (item_hi - 1) / share;
            s.q_head = q_head;
            s.heads_here = heads_here;
            s.b = now.b;
        }
    };

    // One loop for filling the ring and for the steady state, so that its code exists once: a launch fetches every instruction
    // that it runs from memory.
    find_pages();
    load_queries(now);   // before the rows: behind them in the memory system they would come last
    bool begins = true;
    for (int stage = 0, fill = 0, requests = S::kStages; now.index < t1; requests = 1) {
#pragma unroll 1
        for (; requests > 0; --requests) {   // the stage that the step before this one used, or at first all of them
            if (ahead.index < t1) {
                request(fill);
                step<TILE, W>(p, ahead);
                if (ahead.index < t1) {
                    find_pages();
                    if (ahead.tile == 0) prefetch_queries();
                }
            }
            copy_commit();
            fill = fill + 1 == S::kStages ? 0 : fill + 1;
        }
        if (begins) begin_piece();
        copy_wait<S::kStages - 1>();
        __syncwarp();
        products(stage);
        __syncwarp();
        begins = now.tile + 1 == now.r.tiles;
        Place next = now;
        step<TILE, W>(p, next);
        if (begins && next.index < t1) load_queries(next);   // on their way while this piece ends
        if (begins || now.index + 1 == t1) end_piece();
        now = next;
        if (begins) piece_first = now.index;
        stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    copy_wait<0>();

    // ---- (sequence, head)s that several CTAs share: whoever finishes last joins the pieces, in order.  This waits until the
    //      CTA's own list is done, so that its copies never stand still for another's results ----
    __syncthreads();
    if (sh.split[0].c_lo < 0 && sh.split[1].c_lo < 0) return;
    if (tid < 2 && sh.split[tid].c_lo >= 0) {
        auto &s = sh.split[tid];
        const int pieces = s.c_hi - s.c_lo + 1, group = pieces <= S::kMaxJoin ? 0 : (cta - s.c_lo) / kJoinGroup;
        const int g_lo = s.c_lo + group * kJoinGroup;
        const int expected = pieces <= S::kMaxJoin ? pieces : min(kJoinGroup, s.c_hi - g_lo + 1);
        // tickets: [0, max) for an item's first (or only) group, [max, 2 max) for its later ones (their first CTA may start another
        // item's first group), [2 max, 3 max) for the groups' results
        uint32_t *ticket = tickets + (group ? kPagedMaxCtas : 0) + g_lo;
        s.last = NNC_BC(g_lo >= 0 && chunk * (int)gridDim.x + g_lo < kPagedMaxCtas && s.c_hi < (int)gridDim.x, 3204) && take_ticket(ticket, expected);
    }
    __syncthreads();
    // The rows to be joined come into the ring's memory, all of them requested at once (a loop of copies and a loop of sums: this
    // code runs once, so what it costs is fetching it and one trip to memory).
    float2 *ml = reinterpret_cast<float2 *>(comb);                       // [pieces][8 NT]
    float *wgt = reinterpret_cast<float *>(ml + S::kMaxJoin * 8 * NT);      // [8 NT][S::kMaxJoin]
    float2 *tot = reinterpret_cast<float2 *>(wgt + S::kMaxJoin * 8 * NT);   // [8 NT]: M, L
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(smem), ml0 = (uint32_t)__cvta_generic_to_shared(ml);
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
        const int c_lo = sh.split[x].c_lo, c_hi = sh.split[x].c_hi, pieces = c_hi - c_lo + 1;
        if (c_lo < 0 || !sh.split[x].last) continue;
        const int q_head = sh.split[x].q_head, cols = sh.split[x].heads_here * (D / 4), b = sh.split[x].b;
        const bool grouped = pieces > S::kMaxJoin;
        int c0 = grouped ? c_lo + (cta - c_lo) / kJoinGroup * kJoinGroup : c_lo, apart = 1;   // CTAs c0, c0 + apart, ...
        int n = grouped ? min(kJoinGroup, c_hi - c0 + 1) : pieces;
#pragma unroll 1
        for (bool final = !grouped;;) {
            // the first piece of a (sequence, head) lies in its CTA's slot 1, the others in slot 0
            float *const slot_a = part + (size_t)(2 * c0 + (c0 == c_lo ? 1 : 0)) * S::kSlotFloats;
            const float *const slot_b = part + (size_t)(2 * c0) * S::kSlotFloats;   // the i-th from there, i > 0
            const size_t step = (size_t)(2 * apart) * S::kSlotFloats;
            for (int i = tid; i < n * 4 * NT; i += kWarps * 32) {   // 16 bytes: two heads' words
                const int from = i / (4 * NT);
                copy16(ml0 + i * 16, (from ? slot_b + from * step : slot_a) + 8 * NT * D + 4 * (i % (4 * NT)));
            }
            copy_commit();
            const int fit = kWarps * S::kStages * S::kStage / (cols * 16);   // pieces that the ring holds at a time (10 at least)
            if (!NNC_BC(n > 0 && n <= S::kMaxJoin && fit > 0 && c0 + (n - 1) * apart <= c_hi, 3206)) break;
            for (int lo = 0; lo < n; lo += fit) {
                const int hi = min(lo + fit, n);
                for (int col = tid; col < cols; col += kWarps * 32) {
                    uint32_t dst = ring0 + col * 16;
                    const float *src = (lo ? slot_b + lo * step : slot_a) + 4 * col, *next = slot_b + (lo + 1) * step + 4 * col;
#pragma unroll 4
                    for (int i = lo; i < hi; ++i) {
                        copy16(dst, src);
                        dst += cols * 16;
                        src = next;
                        next += step;
                    }
                }
                copy_commit();
                if (lo == 0) {
                    copy_wait<1>();
                    __syncthreads();
                    for (int h = warp; h < 8 * NT; h += kWarps) {   // rows beyond the heads in use weigh what happens to be there
                        const float2 u = lane < n ? ml[lane * 8 * NT + h] : make_float2(-INFINITY, 0.f);
                        const float2 v = lane + 32 < n ? ml[(lane + 32) * 8 * NT + h] : make_float2(-INFINITY, 0.f);
                        const float M = warp_max(fmaxf(u.x, v.x));
                        const float ref = M == -INFINITY ? 0.f : M;
                        const float wu = exp2f(u.x - ref), wv = exp2f(v.x - ref);
                        if (lane < n) wgt[h * S::kMaxJoin + lane] = wu;
                        if (lane + 32 < n) wgt[h * S::kMaxJoin + lane + 32] = wv;
                        const float L = warp_sum(fmaf(wu, u.y, wv * v.y));
                        if (lane == 0) tot[h] = make_float2(M, L);
                    }
                    __syncthreads();
                }
                copy_wait<0>();
                for (int col = tid; col < cols; col += kWarps * 32) {   // every thread reads what it copied itself
                    const int h = col / (D / 4);
                    const float4 *rows = reinterpret_cast<const float4 *>(smem);
                    float4 *slot0 = reinterpret_cast<float4 *>(slot_a) + col;
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (lo > 0) sum = *slot0;   // what the pieces before these gave
                    const float4 from = sum;
#pragma unroll 4
                    for (int i = lo; i < hi; ++i) {
                        const float w = wgt[h * S::kMaxJoin + i];
                        const float4 v = rows[(i - lo) * cols + col];
                        sum.x = fmaf(w, v.x, sum.x); sum.y = fmaf(w, v.y, sum.y); sum.z = fmaf(w, v.z, sum.z); sum.w = fmaf(w, v.w, sum.w);
                    }
                    if (!CODES && !(fabsf((sum.x + sum.y) + (sum.z + sum.w)) < INFINITY)) {   // an infinite piece counts whatever it weighs
                        auto add = [](float w, float v, float sum) { return fabsf(v) == INFINITY ? sum + v : fmaf(w, v, sum); };
                        sum = from;
#pragma unroll 1
                        for (int i = lo; i < hi; ++i) {
                            const float w = wgt[h * S::kMaxJoin + i];
                            const float4 v = rows[(i - lo) * cols + col];
                            sum.x = add(w, v.x, sum.x); sum.y = add(w, v.y, sum.y); sum.z = add(w, v.z, sum.z); sum.w = add(w, v.w, sum.w);
                        }
                    }
                    const float2 ML = tot[h];
                    if (!final || hi < n) {
                        *slot0 = sum;   // this thread alone read that place, and has
                        if (hi == n && col % (D / 4) == 0) *(reinterpret_cast<float2 *>(slot_a + 8 * NT * D) + h) = ML;
                        continue;
                    }
                    const float inv = inverse(ML.y);
                    const long long at = b * p.out_stride + (long long)q_head * D + 4 * col;
                    if constexpr (OUT == NNC_F32) *reinterpret_cast<float4 *>(p.out + at * 4) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
                    else if constexpr (OUT == NNC_BF16)
                        *reinterpret_cast<uint2 *>(p.out + at * 2) = make_uint2(pack_bf16x2(sum.x * inv, sum.y * inv), pack_bf16x2(sum.z * inv, sum.w * inv));
                    else {
                        const __half2 lo2 = __floats2half2_rn(sum.x * inv, sum.y * inv), hi2 = __floats2half2_rn(sum.z * inv, sum.w * inv);
                        *reinterpret_cast<uint2 *>(p.out + at * 2) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo2), *reinterpret_cast<const uint32_t *>(&hi2));
                    }
                    if (p.lse && col % (D / 4) == 0) store_weights((long long)b * (p.c.n_kv * p.group) + q_head + h, ML.x, ML.y);
                }
            }
            __syncthreads();   // what is copied next goes where these weights and rows are
            if (final) break;
            const int groups = (pieces + kJoinGroup - 1) / kJoinGroup;
            if (tid == 0) sh.split[x].last = take_ticket(tickets + 2 * kPagedMaxCtas + c_lo, groups);
            __syncthreads();
            if (!sh.split[x].last) break;
            c0 = c_lo; apart = kJoinGroup; n = groups; final = true;
        }
    }
}

// W::kConcurrent: starts as the preceding kernel's CTAs leave, which let it start after that kernel's own predecessors had ended.  One CTA waits for
// the whole of that kernel in the end, so that whoever waits for this one has waited for both.
template <int D, int NT, int KV, int TYPE, typename W>
__global__ void __launch_bounds__(kWarps * 32, Shape<D, NT, KV, TYPE>::kCtas) attn_paged_kernel(const PagedAttnParams p) {
    attn_paged_cta<D, NT, KV, TYPE, W>(p);
    if constexpr (W::kConcurrent)
        if (blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1) pdl_wait();
}

// the longest list that a table allows: its places are 32-bit numbers
inline bool list_fits(long long most, int tile, int batch, int n_kv, long long *places = nullptr) {
    const long long n = ((most + 15 + tile - 1) / tile + 1) * batch * n_kv;
    if (places) *places = n;
    return n <= 0x3fffffffll;
}

template <int D, int NT, int KV, int TYPE, typename W>
cudaError_t launch_one(const LaunchCtx &lc, const PagedAttnParams &p) {
    typedef Shape<D, NT, KV, TYPE> S;
    static unsigned long long raised = 0;
    auto kern = attn_paged_kernel<D, NT, KV, TYPE, W>;
    cudaError_t e = ensure_dynamic_smem(kern, S::kSmem, &raised);
    if (e != cudaSuccess) return e;
    long long tiles;
    if (!list_fits(W::most(p), S::kTile, p.batch, p.c.n_kv, &tiles)) return cudaErrorInvalidValue;
    long long ctas = (long long)S::kCtas * lc.sm_count;
    if (ctas > kPagedMaxCtas) ctas = kPagedMaxCtas;
    const long long fit = (long long)(p.part_floats / (2 * S::kSlotFloats));
    if (ctas > fit) ctas = fit;
    // Query heads beyond one CTA's go to CTAs of their own that take the same shares at the same time, so that a row that the one
    // has read from memory is in L2 for the others
    ctas /= p.chunks;
    if (ctas > tiles) ctas = tiles;
    if (ctas < 1) ctas = 1;
    LaunchCtx early = lc;
    early.pdl = true;   // the kernel waits for its predecessor itself
    return launch_smem(early, kern, dim3((unsigned)ctas, (unsigned)p.chunks), dim3(kWarps * 32), (size_t)S::kSmem, p);
}

template <typename W, int D, int NT>
cudaError_t launch_typed(const LaunchCtx &lc, const PagedAttnParams &p, int kv, int type) {
    if constexpr (W::kTypeF32)
        if (type == NNC_F32) return kv == NNC_BF16 ? launch_one<D, NT, NNC_BF16, NNC_F32, W>(lc, p) : kv == NNC_F16 ? launch_one<D, NT, NNC_F16, NNC_F32, W>(lc, p) : launch_one<D, NT, NNC_E4M3, NNC_F32, W>(lc, p);
    if (type == NNC_F32) return cudaErrorNotSupported;
    if (kv == NNC_BF16) return launch_one<D, NT, NNC_BF16, NNC_BF16, W>(lc, p);
    if (kv == NNC_F16) return launch_one<D, NT, NNC_F16, NNC_F16, W>(lc, p);
    return type == NNC_BF16 ? launch_one<D, NT, NNC_E4M3, NNC_BF16, W>(lc, p) : launch_one<D, NT, NNC_E4M3, NNC_F16, W>(lc, p);
}

template <typename W> cudaError_t launch_paged_rows(const LaunchCtx &lc, PagedAttnParams p, const nnc_paged_kv &cache, int type) {
    // Query heads in groups of 8.  Two groups as two operands of one CTA share every key and value fragment: 32 x 8192 E4M3 of 64
    // elements, 8 KV heads of 16 query heads: 98 us against 120 with a CTA each.  Not with an odd number of groups, where half of the last
    // pair would be empty (64 x 8192 bf16, 17 heads: 99.9 us in pairs, 90.0 apart), and not where few (sequence, head)s share the whole
    // GPU, whose joins are half as large apart (one of 131072, 16 heads: 31.8 and 26.9 us).
    const int eights = (p.group + 7) / 8;
    const bool two = eights % 2 == 0 && (long long)p.batch * cache.n_kv_heads >= 16;
    p.chunks = two ? eights / 2 : eights;
    if (cache.head_dim == 64) return two ? launch_typed<W, 64, 2>(lc, p, cache.type, type) : launch_typed<W, 64, 1>(lc, p, cache.type, type);
    return two ? launch_typed<W, 128, 2>(lc, p, cache.type, type) : launch_typed<W, 128, 1>(lc, p, cache.type, type);
}

inline PagedAttnParams paged_attn_params(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, void *out, float *lse, int batch,
                                         int n_q_heads, int64_t q_stride, int64_t out_stride, float scale, void *scratch, size_t scratch_bytes) {
    PagedAttnParams p = {};
    p.c = paged_view(cache, lc.status);
    p.q = (const char *)q; p.out = (char *)out; p.lse = lse; p.lens = lens;
    p.tickets = (uint32_t *)scratch;
    p.part = (float *)((char *)scratch + NNC_ATTN_PAGED_TICKET_BYTES);
    p.part_floats = (scratch_bytes - NNC_ATTN_PAGED_TICKET_BYTES) / 4;
    p.q_stride = q_stride; p.out_stride = out_stride;
    p.batch = batch;
    p.group = n_q_heads / cache.n_kv_heads;
    p.scale_log2 = scale * 1.4426950408889634f;
    return p;
}

}  // namespace

}  // namespace nnc
