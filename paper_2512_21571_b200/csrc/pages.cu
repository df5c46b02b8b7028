// Choosing what to attend to in a paged cache: the bounds of every page's keys, the most that a query's product with a key between them
// can be, and the pages of the highest scores.
//
//   bounds[page][head][0 / 1][i] = min / max of k[i] over the page's positions
//   score[b][head][n] = max over the head's queries of sum_i max(q_i lo_i, q_i hi_i),  page n of sequence b
//
// A score reads 4 head_dim bytes a page where the attention reads 4 head_dim a position.  The sum is a product of 2 head_dim
// terms, min(q, 0) . lo + max(q, 0) . hi, so 16 pages and 8 queries are one operand each of the warp-level tensor-core product.
#include <cuda_fp16.h>

#include "paged.cuh"

namespace nnc {

namespace {

constexpr uint32_t kAllLanes = 0xffffffffu;

// ---- bounds ----------------------------------------------------------------------------------------------------------------
//
// A warp takes a page of a KV head: a row is head_dim / 8 pieces of 16 bytes (of codes: / 16), so its lanes hold 2 to 8 rows at a time,
// and what they found is joined at the end.  Bound by reading the keys; minima and maxima of 16-bit values are taken in pairs as they are.

struct BoundsParams {
    PagedView c;
    uint16_t *bounds;
    const int32_t *lens, *first;
    int batch;
};

template <bool BF> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {   // NaN if either is
    uint32_t r;
    if constexpr (BF) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <bool BF> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (BF) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

constexpr int kBoundsWarps = 8;

template <int D, int KV>
__global__ void __launch_bounds__(kBoundsWarps * 32) page_bounds_kernel(const BoundsParams p) {
    constexpr bool CODES = KV == NNC_E4M3, BF = KV != NNC_F16;   // bounds of codes are bf16, which holds every scaled code
    constexpr int kPieces = D * (CODES ? 1 : 2) / 16;            // of a row
    constexpr int kRows = 32 / kPieces;                          // a warp's at a time
    constexpr int kWords = CODES ? 8 : 4;                        // pairs of values of a piece
    constexpr uint32_t kLowest = BF ? 0xff80ff80u : 0xfc00fc00u, kHighest = BF ? 0x7f807f80u : 0x7c007c00u;   // -infinity, infinity
    constexpr int kAhead = 8;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int most = p.c.pages_per_seq << p.c.page_shift, page_size = 1 << p.c.page_shift;
    const int given = p.lens[b], len = max(0, min(given, most)), from = p.first ? max(0, p.first[b]) : 0;
    if (given > most && blockIdx.x == 0 && threadIdx.x == 0) paged_complain(p.c);
    const int c_lo = from >> p.c.page_shift, c_hi = (len + page_size - 1) >> p.c.page_shift;
    if (from >= len) return;
    const long long units = (long long)(c_hi - c_lo) * p.c.n_kv;
    const int piece = lane % kPieces, r0 = lane / kPieces;
    for (long long unit = (long long)blockIdx.x * kBoundsWarps + warp; unit < units; unit += (long long)gridDim.x * kBoundsWarps) {
        const int column = c_lo + (int)(unit / p.c.n_kv), head = (int)(unit % p.c.n_kv);
        if (!NNC_BC(column < p.c.pages_per_seq && b < p.batch, 3401)) continue;
        const int page = p.c.table[(long long)b * p.c.pages_per_seq + column];
        if ((unsigned)page >= (unsigned)p.c.n_pages) {
            if (lane == 0) paged_complain(p.c);
            continue;
        }
        const int rows = min(page_size, len - (column << p.c.page_shift));
        const long long row0 = paged_row(p.c, page, head, 0);
        const char *src = p.c.k + row0 * (D * (CODES ? 1 : 2)) + piece * 16;
        uint32_t lo[kWords], hi[kWords];
#pragma unroll
        for (int w = 0; w < kWords; ++w) { lo[w] = kHighest; hi[w] = kLowest; }
        auto take = [&](uint4 x, int row) {
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (!CODES) {
                    lo[w] = min2<BF>(lo[w], in[w]);
                    hi[w] = max2<BF>(hi[w], in[w]);
                } else {
                    const float scale = scale_from_byte(p.c.k_scale[row0 + row]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t h = e4m3x2_to_f16x2(in[w] >> (16 * e) & 0xffffu);
                        const __half2 f = *reinterpret_cast<const __half2 *>(&h);
                        const uint32_t v = pack_bf16x2(__low2float(f) * scale, __high2float(f) * scale);
                        lo[2 * w + e] = min2<BF>(lo[2 * w + e], v);
                        hi[2 * w + e] = max2<BF>(hi[2 * w + e], v);
                    }
                }
            }
        };
        for (int at = r0; at < rows; at += kAhead * kRows) {
            uint4 x[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (at + i * kRows < rows) x[i] = ldg_stream(src + (long long)(at + i * kRows) * (D * (CODES ? 1 : 2)));
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (at + i * kRows < rows) take(x[i], at + i * kRows);
        }
#pragma unroll
        for (int o = kPieces; o < 32; o <<= 1)
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                lo[w] = min2<BF>(lo[w], __shfl_xor_sync(kAllLanes, lo[w], o));
                hi[w] = max2<BF>(hi[w], __shfl_xor_sync(kAllLanes, hi[w], o));
            }
        if (r0 == 0) {
            uint4 *dst = reinterpret_cast<uint4 *>(p.bounds + ((long long)page * p.c.n_kv + head) * (2 * D)) + piece * (kWords / 4);
#pragma unroll
            for (int w = 0; w < kWords; w += 4) {
                dst[w / 4] = make_uint4(lo[w], lo[w + 1], lo[w + 2], lo[w + 3]);
                dst[w / 4 + D / 8] = make_uint4(hi[w], hi[w + 1], hi[w + 2], hi[w + 3]);
            }
        }
    }
}

// ---- scores ----------------------------------------------------------------------------------------------------------------
//
// Lane (g8, t4) of a warp loads 16 bytes of the bounds of pages g8 and g8 + 8 at a time: eight neighbouring elements, which stand in the
// columns 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9 of two steps of the product; the queries' elements are laid out the same way in shared memory.
// So nothing is staged, and a warp has 8 KB (of 128-element heads) on their way at once.

constexpr int kScoreWarps = 4;

struct ScoreParams {
    PagedView c;
    const char *q;
    const uint16_t *bounds;
    const int32_t *lens;
    float *scores;
    long long q_stride;
    int batch, group, splits;
};

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <bool BF> __device__ __forceinline__ void mma_step(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
    if constexpr (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}

// BF: bounds are bf16; TYPE: the queries'; TERMS of BF's type make a query exactly (fp32 ones: to 24 or 22 bits)
template <int D, bool BF, int TYPE, int TERMS>
__global__ void __launch_bounds__(kScoreWarps * 32) score_pages_kernel(const ScoreParams p) {
    constexpr int kSteps = 2 * D / 16;   // of the product: D / 16 of the lower bounds, as many of the upper
    extern __shared__ __align__(16) uint2 operand[];   // [groups of 8 queries][TERMS][kSteps][32 lanes]
    __shared__ float undo[1024];   // fp16 terms of fp32 queries: what every query was multiplied by, inverted
    constexpr bool SCALED = !BF && TYPE == NNC_F32;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3;
    const int split = blockIdx.x % p.splits, head = blockIdx.x / p.splits % p.c.n_kv, b = blockIdx.x / p.splits / p.c.n_kv;
    const int most = p.c.pages_per_seq << p.c.page_shift;
    const int given = p.lens[b], len = max(0, min(given, most));
    if (given > most && split == 0 && head == 0 && tid == 0) paged_complain(p.c);
    const int pages = (len + (1 << p.c.page_shift) - 1) >> p.c.page_shift, columns = p.c.pages_per_seq;
    float *const scores = p.scores + ((long long)b * p.c.n_kv + head) * columns;
    const int chunks = (p.group + 7) / 8;
    // ---- the queries, as the product's second operand ----
    auto query = [&](int g, int i) -> float {
        if (g >= p.group) return 0.f;
        const long long at = b * p.q_stride + ((long long)head * p.group + g) * D + i;
        if constexpr (TYPE == NNC_F32) return reinterpret_cast<const float *>(p.q)[at];
        else if constexpr (TYPE == NNC_BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(p.q)[at]);
        else return __half2float(reinterpret_cast<const __half *>(p.q)[at]);
    };
    if constexpr (SCALED) {   // a query times the power of two that brings its largest magnitude into [2^14, 2^15)
        for (int g = warp; g < chunks * 8; g += kScoreWarps) {
            float top = 0.f;
            for (int i = lane; i < D; i += 32) top = fmaxf(top, fabsf(query(g, i)));
            top = warp_max(top);
            const int e8 = (int)(__float_as_uint(top) >> 23);
            const int up8 = (top == 0.f || e8 >= 255) ? 127 : min(268 - e8, 253);
            if (lane == 0) undo[g] = __uint_as_float((uint32_t)(254 - up8) << 23);
        }
        __syncthreads();
    }
    for (int i = tid; i < chunks * (kSteps / 2) * 32; i += kScoreWarps * 32) {
        const int l = i & 31, s = i / 32 % (kSteps / 2), chunk = i / 32 / (kSteps / 2);
        const int g = chunk * 8 + (l >> 2), from = 32 * (s / 2) + 8 * (l & 3) + 4 * (s & 1);   // step s: half of the lanes' 16-byte pieces
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = query(g, from + e);
        if constexpr (SCALED) {
            const float up = 1.f / undo[g];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= up;
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            uint32_t w[2][2];   // [negative, positive part][pair]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint32_t both;
                if constexpr (BF) {
                    both = pack_bf16x2(x[2 * e], x[2 * e + 1]);
                    x[2 * e] -= bf16_lo(both); x[2 * e + 1] -= bf16_hi(both);
                } else {
                    const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
                    both = *reinterpret_cast<const uint32_t *>(&h);
                    x[2 * e] -= __low2float(h); x[2 * e + 1] -= __high2float(h);
                }
                w[0][e] = w[1][e] = both;
            }
            // the sign of the query itself, not of a term, says which bound it meets
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t half = 0xffffu << (16 * (e & 1));
                w[query(g, from + e) < 0.f ? 1 : 0][e / 2] &= ~half;
            }
            uint2 *dst = operand + ((chunk * TERMS + t) * kSteps + s) * 32 + l;
            dst[0] = make_uint2(w[0][0], w[0][1]);
            dst[(kSteps / 2) * 32] = make_uint2(w[1][0], w[1][1]);
        }
    }
    __syncthreads();
    // ---- 16 pages at a time ----
    for (int n0 = (split * kScoreWarps + warp) * 16; n0 < columns; n0 += p.splits * kScoreWarps * 16) {
        const int mine = n0 + (lane & 15);
        int page = -1;
        if (mine < pages) {
            page = p.c.table[(long long)b * columns + mine];
            if ((unsigned)page >= (unsigned)p.c.n_pages || !NNC_BC(b < p.batch && head < p.c.n_kv, 3402)) { paged_complain(p.c); page = -1; }
        }
        float best = -INFINITY;   // of page n0 + lane % 16
        if (n0 < pages) {
            uint4 x[2][kSteps / 2];   // pieces of pages g8 and g8 + 8
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = __shfl_sync(kAllLanes, page, g8 + 8 * r);
                const uint4 *src = reinterpret_cast<const uint4 *>(p.bounds + ((long long)max(at, 0) * p.c.n_kv + head) * (2 * D)) + t4;
#pragma unroll
                for (int s = 0; s < kSteps / 2; ++s) x[r][s] = ldg_stream(src + 4 * s);
            }
            float top[2] = {-INFINITY, -INFINITY};
            for (int chunk = 0; chunk < chunks; ++chunk) {
                constexpr int kSums = TERMS > 1 ? 3 : 2;   // lower bounds, upper bounds, lower terms
                float acc[kSums][4];
#pragma unroll
                for (int i = 0; i < kSums; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
                const uint2 *w = operand + chunk * TERMS * kSteps * 32 + lane;
#pragma unroll
                for (int s = 0; s < kSteps / 2; ++s)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        float (&sum)[4] = acc[t ? 2 : s < kSteps / 4 ? 0 : 1];
                        mma_step<BF>(sum, x[0][s].x, x[1][s].x, x[0][s].y, x[1][s].y, w[(t * kSteps + 2 * s) * 32]);
                        mma_step<BF>(sum, x[0][s].z, x[1][s].z, x[0][s].w, x[1][s].w, w[(t * kSteps + 2 * s + 1) * 32]);
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // pages g8, g8 + 8; queries 2 t4, 2 t4 + 1
                    const int g = chunk * 8 + 2 * t4 + (e & 1);
                    float s = acc[0][e] + acc[1][e];
                    if constexpr (TERMS > 1) s += fabsf(s) == INFINITY ? 0.f : acc[2][e];   // (an infinity is the first terms')
                    if constexpr (SCALED) s *= undo[g];
                    if (g < p.group) top[e >> 1] = max_nan(top[e >> 1], s);
                }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = max_nan(top[r], __shfl_xor_sync(kAllLanes, top[r], 1));
                top[r] = max_nan(top[r], __shfl_xor_sync(kAllLanes, top[r], 2));
            }
            const float low = __shfl_sync(kAllLanes, top[0], (lane & 7) * 4), high = __shfl_sync(kAllLanes, top[1], (lane & 7) * 4);
            best = page < 0 ? -INFINITY : lane & 8 ? high : low;
        }
        if (lane < 16 && mine < columns) scores[mine] = best;
    }
}

// ---- selection ---------------------------------------------------------------------------------------------------------------
//
// A CTA a row.  Scores become whole numbers of the same order; four passes over 8 bits each find the n-th largest (a histogram, and the
// bin that the n-th falls into), a fifth writes the indices of what is above it, and of as many of its equals as are missing, in order.

constexpr int kSelectThreads = 512;

struct SelectParams {
    const float *scores;
    const int32_t *lens;
    int32_t *pages, *counts;
    int n_kv, columns, page_shift, n, first, last, kept;   // kept: the row's numbers fit in shared memory
};

__global__ void __launch_bounds__(kSelectThreads) select_pages_kernel(const SelectParams p) {
    extern __shared__ uint32_t row_keys[];
    __shared__ uint32_t histogram[256];
    __shared__ uint32_t chosen_bin, left;
    __shared__ uint2 sums[kSelectThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x;
    const int len = p.lens[row / p.n_kv];
    const int pages = len <= 0 ? 0 : min((int)(((long long)len + (1 << p.page_shift) - 1) >> p.page_shift), p.columns);
    int32_t *const out = p.pages + row * p.n;
    const int count = min(pages, p.n);
    if (tid == 0) p.counts[row] = count;
    for (int i = count + tid; i < p.n; i += kSelectThreads) out[i] = -1;
    if (pages <= p.n) {
        for (int i = tid; i < count; i += kSelectThreads) out[i] = i;
        return;
    }
    const float *const scores = p.scores + row * p.columns;
    auto key_of = [&](int i) -> uint32_t {
        if (i < p.first || i >= pages - p.last) return 0xffffffffu;
        const float x = scores[i] + 0.f;   // (-0 is 0)
        if (x != x) return 0xfffffffeu;    // NaN: above every number
        const uint32_t u = __float_as_uint(x);
        return u & 0x80000000u ? ~u : u | 0x80000000u;
    };
    if (p.kept)
        for (int i = tid; i < pages; i += kSelectThreads) row_keys[i] = key_of(i);
    auto key = [&](int i) { return p.kept ? row_keys[i] : key_of(i); };   // (a thread reads what it wrote itself)
    uint32_t above = 0, need = p.n;   // above: the bits of the n-th largest that are known; need: how many of those that share them
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) histogram[i] = 0;
        __syncthreads();
        for (int i = tid; i < pages; i += kSelectThreads) {
            const uint32_t k = key(i);
            if (shift == 24 || (k >> (shift + 8)) == (above >> (shift + 8))) atomicAdd(&histogram[k >> shift & 255u], 1u);
        }
        __syncthreads();
        if (warp == 0) {   // lane l holds bins 255 - 8 l .. 248 - 8 l, the highest first
            uint32_t n[8], sum = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) { n[j] = histogram[255 - 8 * lane - j]; sum += n[j]; }
            uint32_t before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(kAllLanes, before, o);
                if (lane >= o) before += x;
            }
            before -= sum;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (before < need && need <= before + n[j]) { chosen_bin = 255 - 8 * lane - j; left = need - before; }
                before += n[j];
            }
        }
        __syncthreads();
        above |= chosen_bin << shift;
        need = left;
    }
    // ---- in order: what lies above, and the first `need` of the equals ----
    uint32_t done_above = 0, done_equal = 0;
    for (int i0 = 0; i0 < pages; i0 += kSelectThreads) {
        const int i = i0 + tid;
        const uint32_t k = i < pages ? key(i) : 0u;
        const bool is_above = i < pages && k > above, is_equal = i < pages && k == above;
        const uint32_t va = __ballot_sync(kAllLanes, is_above), ve = __ballot_sync(kAllLanes, is_equal), before = (1u << lane) - 1u;
        if (lane == 0) sums[warp] = make_uint2(__popc(va), __popc(ve));
        __syncthreads();
        uint32_t a = done_above, e = done_equal;
        for (int w = 0; w < kSelectThreads / 32; ++w) {
            const uint2 s = sums[w];
            if (w < warp) { a += s.x; e += s.y; }
            done_above += s.x; done_equal += s.y;
        }
        __syncthreads();
        a += __popc(va & before);
        e += __popc(ve & before);
        if (is_above || (is_equal && e < need)) {
            const uint32_t at = a + min(e, need);
            if (NNC_BC(at < (uint32_t)p.n, 3403)) out[at] = i;
        }
    }
}

template <int D> cudaError_t launch_bounds_of(const LaunchCtx &lc, const BoundsParams &p, int kv, dim3 grid) {
    const dim3 block(kBoundsWarps * 32);
    if (kv == NNC_BF16) return launch(lc, page_bounds_kernel<D, NNC_BF16>, grid, block, p);
    if (kv == NNC_F16) return launch(lc, page_bounds_kernel<D, NNC_F16>, grid, block, p);
    return launch(lc, page_bounds_kernel<D, NNC_E4M3>, grid, block, p);
}

template <int D, bool BF, int TYPE, int TERMS> cudaError_t launch_score_of(const LaunchCtx &lc, const ScoreParams &p, dim3 grid) {
    const int smem = (p.group + 7) / 8 * TERMS * (2 * D / 16) * 32 * (int)sizeof(uint2);
    static unsigned long long raised = 0;
    if (smem > 200 << 10) return cudaErrorInvalidValue;
    if (smem > 32 << 10)
        if (cudaError_t e = ensure_dynamic_smem(score_pages_kernel<D, BF, TYPE, TERMS>, 200 << 10, &raised); e != cudaSuccess) return e;
    return launch_smem(lc, score_pages_kernel<D, BF, TYPE, TERMS>, grid, dim3(kScoreWarps * 32), (size_t)smem, p);
}

template <int D> cudaError_t launch_score_typed(const LaunchCtx &lc, const ScoreParams &p, int kv, int type, dim3 grid) {
    if (kv == NNC_F16) return type == NNC_F32 ? launch_score_of<D, false, NNC_F32, 2>(lc, p, grid) : launch_score_of<D, false, NNC_F16, 1>(lc, p, grid);
    if (type == NNC_F32) return launch_score_of<D, true, NNC_F32, 3>(lc, p, grid);
    return type == NNC_BF16 ? launch_score_of<D, true, NNC_BF16, 1>(lc, p, grid) : launch_score_of<D, true, NNC_F16, 2>(lc, p, grid);
}

}  // namespace

cudaError_t launch_page_bounds(const LaunchCtx &lc, const nnc_paged_kv &cache, void *bounds, const int32_t *lens, const int32_t *first, int batch) {
    BoundsParams p;
    p.c = paged_view(cache, lc.status);
    p.bounds = (uint16_t *)bounds; p.lens = lens; p.first = first; p.batch = batch;
    const long long most = ((long long)cache.pages_per_seq * cache.n_kv_heads + kBoundsWarps - 1) / kBoundsWarps;
    long long ctas = (8ll * lc.sm_count + batch - 1) / batch;   // lengths are the device's: as many as fill it if all sequences are alike
    if (ctas > most) ctas = most;
    LaunchCtx early = lc;
    early.pdl = true;
    const dim3 grid((unsigned)ctas, (unsigned)batch);
    return cache.head_dim == 64 ? launch_bounds_of<64>(early, p, cache.type, grid) : launch_bounds_of<128>(early, p, cache.type, grid);
}

cudaError_t launch_score_pages(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const void *bounds, const int32_t *lens, float *scores,
                               int type, int batch, int n_q_heads, int64_t q_stride) {
    ScoreParams p;
    p.c = paged_view(cache, lc.status);
    p.q = (const char *)q; p.bounds = (const uint16_t *)bounds; p.lens = lens; p.scores = scores;
    p.q_stride = q_stride; p.batch = batch; p.group = n_q_heads / cache.n_kv_heads;
    const long long rows = (long long)batch * cache.n_kv_heads;
    const long long most = (cache.pages_per_seq + 16 * kScoreWarps - 1) / (16 * kScoreWarps);
    long long splits = (8ll * lc.sm_count + rows - 1) / rows;
    if (splits > most) splits = most;
    p.splits = (int)splits;
    if (rows * splits > 0x7fffffff) return cudaErrorInvalidValue;
    LaunchCtx early = lc;
    early.pdl = true;
    const dim3 grid((unsigned)(rows * splits));
    return cache.head_dim == 64 ? launch_score_typed<64>(early, p, cache.type, type, grid) : launch_score_typed<128>(early, p, cache.type, type, grid);
}

cudaError_t launch_select_pages(const LaunchCtx &lc, const float *scores, const int32_t *lens, int32_t *pages, int32_t *counts, int batch, int n_kv,
                                int columns, int page_size, int n, int first, int last) {
    SelectParams p;
    p.scores = scores; p.lens = lens; p.pages = pages; p.counts = counts;
    p.n_kv = n_kv; p.columns = columns; p.page_shift = __builtin_ctz((unsigned)page_size);
    p.n = n; p.first = first; p.last = last;
    p.kept = columns <= (160 << 10) / 4;
    const size_t smem = p.kept ? (size_t)columns * 4 : 0;
    static unsigned long long raised = 0;
    if (smem > 32 << 10)
        if (cudaError_t e = ensure_dynamic_smem(select_pages_kernel, 160 << 10, &raised); e != cudaSuccess) return e;
    LaunchCtx early = lc;
    early.pdl = true;
    return launch_smem(early, select_pages_kernel, dim3((unsigned)((long long)batch * n_kv)), dim3(kSelectThreads), smem, p);
}

}  // namespace nnc
