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
// and what they found is joined at the end.  Bound by reading the keys (4 prompts of 16384 positions, 8 heads of 128: 22.2 us, 95 % of a plain copy's
// rate), or by launch, length, page and rows one after the other (a page each of 48 sequences: 5.5 us); minima and maxima of 16-bit values are
// taken in pairs as they are.

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
        if (!NNC_BC(column < p.c.pages_per_seq && b < p.batch, 3801)) continue;
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
// So nothing is staged, and a warp has 8 KB (of 128-element heads) on their way at once.  Bound by reading the bounds (32 sequences of 2048 pages, 8
// heads: 26.2 us, 79 % of a plain copy's rate), or by the queries' layout and one trip to memory (one of 4096 pages, fp32 queries: 6.3 us).

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
    __shared__ float undo[kMaxScoredGroup];   // fp16 terms of fp32 queries: what every query was multiplied by, inverted
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
        uint32_t minus[2] = {0u, 0u};   // all bits of negative elements, in pairs
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = query(g, from + e);
            if (x[e] < 0.f) minus[e / 2] |= 0xffffu << (16 * (e & 1));
        }
        if constexpr (SCALED) {
            const float up = 1.f / undo[g];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= up;
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            uint32_t both[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if constexpr (BF) {
                    both[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
                    x[2 * e] -= bf16_lo(both[e]); x[2 * e + 1] -= bf16_hi(both[e]);
                } else {
                    const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
                    both[e] = *reinterpret_cast<const uint32_t *>(&h);
                    x[2 * e] -= __low2float(h); x[2 * e + 1] -= __high2float(h);
                }
            }
            // the sign of the query itself, not of a term, says which bound it meets
            uint2 *dst = operand + ((chunk * TERMS + t) * kSteps + s) * 32 + l;
            dst[0] = make_uint2(both[0] & minus[0], both[1] & minus[1]);
            dst[(kSteps / 2) * 32] = make_uint2(both[0] & ~minus[0], both[1] & ~minus[1]);
        }
    }
    __syncthreads();
    // ---- 16 pages at a time ----
    for (int n0 = (split * kScoreWarps + warp) * 16; n0 < columns; n0 += p.splits * kScoreWarps * 16) {
        const int mine = n0 + (lane & 15);
        int page = -1;
        if (mine < pages) {
            page = p.c.table[(long long)b * columns + mine];
            if ((unsigned)page >= (unsigned)p.c.n_pages || !NNC_BC(b < p.batch && head < p.c.n_kv, 3802)) { paged_complain(p.c); page = -1; }
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
                float acc[2][TERMS][4];   // lower bounds, upper bounds: a chain of products each
#pragma unroll
                for (int i = 0; i < 2 * TERMS; ++i) acc[i & 1][i >> 1][0] = acc[i & 1][i >> 1][1] = acc[i & 1][i >> 1][2] = acc[i & 1][i >> 1][3] = 0.f;
                const uint2 *w = operand + chunk * TERMS * kSteps * 32 + lane;
#pragma unroll
                for (int s = 0; s < kSteps / 4; ++s)
#pragma unroll
                    for (int side = 0; side < 2; ++side)
#pragma unroll
                        for (int t = 0; t < TERMS; ++t) {
                            const int load = side * (kSteps / 4) + s;
                            mma_step<BF>(acc[side][t], x[0][load].x, x[1][load].x, x[0][load].y, x[1][load].y, w[(t * kSteps + 2 * load) * 32]);
                            mma_step<BF>(acc[side][t], x[0][load].z, x[1][load].z, x[0][load].w, x[1][load].w, w[(t * kSteps + 2 * load + 1) * 32]);
                        }
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // pages g8, g8 + 8; queries 2 t4, 2 t4 + 1
                    const int g = chunk * 8 + 2 * t4 + (e & 1);
                    float s = acc[0][0][e] + acc[1][0][e];
                    if constexpr (TERMS > 1) {
                        float rest = 0.f;
#pragma unroll
                        for (int t = TERMS - 1; t > 0; --t) rest += acc[0][t][e] + acc[1][t][e];
                        s += fabsf(s) == INFINITY ? 0.f : rest;   // (an infinity is the first terms')
                    }
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
// A CTA a row.  Scores become whole numbers of the same order, in registers (up to 8704 pages) or in shared memory.  A histogram of 2048 equal
// parts of their range tells the part that the n-th largest lies in; that part is divided again, until all of it is wanted (scores of one
// batch are spread well enough for one or two rounds) or its numbers are one.  Then the indices of what lies above, and of as many of the
// equals as are missing, are written in order.  Bound by its chain of barriers: 5.4 us for 8 rows of 4097, 5.5 for 256 of 2049, the host's call among
// them.  (By digits of 8 bits: 10.1 and 11.9, as most scores have the highest digit in common; bit by bit, with a vote each: 9.5 and 10.5.)

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kSelectBins = 2048;

struct SelectParams {
    const float *scores;
    const int32_t *lens;
    int32_t *pages, *counts;
    int n_kv, columns, page_shift, n, first, last, kept;   // kept: the row's numbers fit in shared memory
};

// ITEMS: numbers of a thread, in registers; 0: any number, in shared memory if p.kept, otherwise made again from the scores each time
template <int ITEMS>
__global__ void __launch_bounds__(kSelectThreads) select_pages_kernel(const SelectParams p) {
    extern __shared__ uint32_t row_keys[];
    constexpr int kChunks = ITEMS ? ITEMS : 16;                  // runs of kSelectThreads pages that are counted at a time
    constexpr int kEach = (kChunks * kSelectWarps + 31) / 32;    // counts of a lane that adds them up
    __shared__ __align__(16) uint32_t histogram[kSelectBins];    // read and cleared four at a time
    __shared__ uint2 sums[kEach * 32];                           // of a warp's pages of a run: above, equal; then of what came before
    __shared__ uint2 all_sums;
    __shared__ uint32_t most[kSelectWarps], least[kSelectWarps], found[3];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x;
    const float *const scores = p.scores + row * p.columns;
    const int len = p.lens[row / p.n_kv];
    float early[ITEMS ? ITEMS : 1];                              // scores, on their way with the length
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (tid + j * kSelectThreads < p.columns) early[j] = scores[tid + j * kSelectThreads];
    for (int i = tid; i < kSelectBins; i += kSelectThreads) histogram[i] = 0;
    const int pages = len <= 0 ? 0 : min((int)(((long long)len + (1 << p.page_shift) - 1) >> p.page_shift), p.columns);
    int32_t *const out = p.pages + row * p.n;
    const int count = min(pages, p.n);
    if (tid == 0) p.counts[row] = count;
    for (int i = count + tid; i < p.n; i += kSelectThreads) out[i] = -1;
    if (pages <= p.n) {
        for (int i = tid; i < count; i += kSelectThreads) out[i] = i;
        return;
    }
    auto key_of = [&](int i, float score) -> uint32_t {
        if (i < p.first || i >= pages - p.last) return 0xffffffffu;
        const float x = score + 0.f;       // (-0 is 0)
        if (x != x) return 0xfffffffeu;    // NaN: above every number
        const uint32_t u = __float_as_uint(x);
        return u & 0x80000000u ? ~u : u | 0x80000000u;
    };
    uint32_t mine[ITEMS ? ITEMS : 1], top = 0, low = 0xffffffffu;
    auto widen = [&](uint32_t k) {   // the range of the scores; pages that are in anyway do not count
        if (k != 0xffffffffu) { top = max(top, k); low = min(low, k); }
    };
    if constexpr (ITEMS > 0) {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const int i = tid + j * kSelectThreads;
            mine[j] = i < pages ? key_of(i, early[j]) : 0u;      // (0 is less than any number's key)
            if (i < pages) widen(mine[j]);
        }
    } else {
        for (int i = tid; i < pages; i += kSelectThreads) {
            const uint32_t k = key_of(i, scores[i]);
            if (p.kept) row_keys[i] = k;   // (a thread reads what it wrote itself)
            widen(k);
        }
    }
    auto each = [&](auto f) {   // this thread's keys; 0 for none
        if constexpr (ITEMS > 0) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) f(mine[j]);
        } else {
            for (int i = tid; i < pages; i += kSelectThreads) f(p.kept ? row_keys[i] : key_of(i, scores[i]));
        }
    };
    top = __reduce_max_sync(kAllLanes, top);
    low = __reduce_min_sync(kAllLanes, low);
    if (lane == 0) { most[warp] = top; least[warp] = low; }
    __syncthreads();
    top = __reduce_max_sync(kAllLanes, most[lane & (kSelectWarps - 1)]);
    low = __reduce_min_sync(kAllLanes, least[lane & (kSelectWarps - 1)]);
    // wanted: how many of the numbers in [low, low + span] (pages that are in anyway lie above: first + last <= n < pages)
    uint32_t need = p.n - (p.first + p.last), span = top - low;
    bool all = need == 0;            // all numbers from `low` on are wanted (with need == 0: none below the pages that are in anyway)
    if (all) low = 0xffffffffu;
#pragma unroll 1
    while (!all && span > 0) {
        const int shift = max(0, 21 - __clz(span));   // span >> shift < 2048
        each([&](uint32_t k) {
            if (k - low <= span && k != 0xffffffffu && k >= low) atomicAdd(&histogram[(k - low) >> shift], 1u);
        });
        __syncthreads();
        // four parts a thread, the highest first
        uint4 part = *reinterpret_cast<const uint4 *>(histogram + kSelectBins - 4 - 4 * tid);
        const uint32_t n4[4] = {part.w, part.z, part.y, part.x}, sum = part.x + part.y + part.z + part.w;
        uint32_t before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kAllLanes, before, o);
            if (lane >= o) before += x;
        }
        if (lane == 31) most[warp] = before;
        __syncthreads();
        const uint32_t others = lane < warp ? most[lane & (kSelectWarps - 1)] : 0u;   // (warp <= 15)
        before += __reduce_add_sync(kAllLanes, others) - sum;
        if (before < need && need <= before + sum) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (before < need && need <= before + n4[j]) { found[0] = kSelectBins - 1 - 4 * tid - j; found[1] = need - before; found[2] = n4[j]; }
                before += n4[j];
            }
        }
        *reinterpret_cast<uint4 *>(histogram + kSelectBins - 4 - 4 * tid) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        low += found[0] << shift;
        span = (1u << shift) - 1u;
        need = found[1];
        all = found[2] == need;
    }
    // Wanted: everything above `nth`; where that is not enough, the first `need` of its equals.
    const uint32_t nth = all ? low - 1u : low;
    if (all) need = 0;
    // ---- in order ----
    uint2 done = make_uint2(0u, 0u);
    for (int i0 = 0; i0 < pages; i0 += kChunks * kSelectThreads) {
        uint32_t va[kChunks], ve[kChunks];
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int i = i0 + j * kSelectThreads + tid;
            uint32_t k = 0;
            if constexpr (ITEMS > 0) k = mine[j];
            else if (i < pages) k = p.kept ? row_keys[i] : key_of(i, scores[i]);
            va[j] = __ballot_sync(kAllLanes, i < pages && k > nth);
            ve[j] = __ballot_sync(kAllLanes, i < pages && k == nth);
            if (lane == 0) sums[j * kSelectWarps + warp] = make_uint2(__popc(va[j]), __popc(ve[j]));
        }
        __syncthreads();
        if (warp == 0) {   // what comes before each: a lane adds up its own, the warp its lanes
            uint2 s[kEach], own = make_uint2(0u, 0u);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                s[j] = lane * kEach + j < kChunks * kSelectWarps ? sums[lane * kEach + j] : make_uint2(0u, 0u);
                own.x += s[j].x; own.y += s[j].y;
            }
            uint2 x = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t a = __shfl_up_sync(kAllLanes, x.x, o), e = __shfl_up_sync(kAllLanes, x.y, o);
                if (lane >= o) { x.x += a; x.y += e; }
            }
            if (lane == 31) all_sums = make_uint2(done.x + x.x, done.y + x.y);
            x.x += done.x - own.x; x.y += done.y - own.y;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                sums[lane * kEach + j] = x;
                x.x += s[j].x; x.y += s[j].y;
            }
        }
        __syncthreads();
        done = all_sums;
        const uint32_t before = (1u << lane) - 1u;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const uint2 s = sums[j * kSelectWarps + warp];
            const uint32_t e = s.y + __popc(ve[j] & before);
            if ((va[j] | (e < need ? ve[j] : 0u)) >> lane & 1u) {
                const uint32_t at = s.x + __popc(va[j] & before) + min(e, need);
                if (NNC_BC(at < (uint32_t)p.n, 3803)) out[at] = i0 + j * kSelectThreads + tid;
            }
        }
        __syncthreads();
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
    LaunchCtx early = lc;
    early.pdl = true;
    const dim3 grid((unsigned)((long long)batch * n_kv)), block(kSelectThreads);
    p.kept = 1;
    // Numbers of a thread in registers: 2, and one more than 4, 8 and 16, as tables of 2^k pages often have a column to spare.  us for 8 and 256 rows, at both ends
    // of each form's widths: 512 and 1024 columns 5.5 and 5.6 | 1025 5.4 and 5.5, 2560 5.1 and 5.6 | 2561 5.1 and 9.4, 4608 5.5 and 9.9 | 4609 6.6 and 13.1,
    // 8704 8.0 and 14.5.  (16 instead of 17: 3 % less up to 8192, 12.3 and 24.8 for 8193.)  In shared memory: 8705 12.7 and 25.8, 16384 19.4 and 36.4,
    // 40960 42 and 81.  Made again from the scores each time: 40961 60 and 111, 131072 307 and 699.
    if (columns <= 2 * kSelectThreads) return launch(early, select_pages_kernel<2>, grid, block, p);
    if (columns <= 5 * kSelectThreads) return launch(early, select_pages_kernel<5>, grid, block, p);
    if (columns <= 9 * kSelectThreads) return launch(early, select_pages_kernel<9>, grid, block, p);
    if (columns <= 17 * kSelectThreads) return launch(early, select_pages_kernel<17>, grid, block, p);
    p.kept = columns <= (160 << 10) / 4;
    const size_t smem = p.kept ? (size_t)columns * 4 : 0;
    static unsigned long long raised = 0;
    if (smem > 32 << 10)
        if (cudaError_t e = ensure_dynamic_smem(select_pages_kernel<0>, 160 << 10, &raised); e != cudaSuccess) return e;
    return launch_smem(early, select_pages_kernel<0>, grid, block, smem, p);
}

}  // namespace nnc
