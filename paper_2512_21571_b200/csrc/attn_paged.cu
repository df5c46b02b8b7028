// Attention of one new token per sequence over a paged key-value cache, sequences of any lengths.
//
//   s_n = scale q.k_n,  o = sum_n exp(s_n - m) v_n / sum_n exp(s_n - m),  n over the attended positions
//
// Bound by reading every attended key and value row once.  How it gets there:
//   - The work is the list of tiles (4 * PB positions of one sequence and KV head; its query heads ride along in groups of
//     up to 16), in the order sequence, head, position.  The lengths live on the device, so every CTA adds up the list
//     itself and takes an equal contiguous share; two CTAs are resident per SM.  A share may end inside a (sequence, head):
//     such pieces leave partial results (m, l, o~) that the CTA finishing last joins in list order (a ticket word;
//     nobody waits), so the result does not depend on who was last.
//   - A warp owns PB positions of every tile and runs its own ring of shared-memory stages, filled by 16-byte asynchronous
//     copies that run ahead across heads and sequences; no barrier in the steady state.  Rows outside the attended
//     range are filled with zeros instead of being read, so nothing stored there can reach a product.
//   - Both products run on the warp-level tensor-core path in transposed form: S^T = K Q^T and O^T = V^T P^T, so 16
//     positions (16 head-dimension elements) fill the 16-row operand and 8 query heads are the 8-column operand.  A
//     tcgen05 tile would be 128 rows for the same 8 columns and wants its operand staged in its own layout, E4M3 codes
//     converted first; the products take under a quarter of the issue slots at full memory rate, so that buys nothing.
//   - E4M3 codes are fp16 values exactly; key scales multiply the scores, value scales (powers of two) are added to the
//     exponents of the probabilities that weigh the codes, so no code is ever multiplied by a scale.
// Numerics: scores, maxima, sums and outputs are fp32.  Queries enter exactly (16-bit types) or as enough terms for fp32 (three
// bf16 or two fp16 terms); probabilities as two bf16 or fp16 terms (three bf16 for fp32 results): 2^-17 or better, below the
// rounding of a 16-bit result, where one bf16 term would be as large as it.
#include <cuda_fp16.h>

#include "paged.cuh"

namespace nnc {

namespace {

constexpr int kWarps = 4;

struct PagedAttnParams {
    PagedView c;
    const char *q;
    char *out;
    float *lse;
    const int32_t *lens;
    float *part;
    uint32_t *tickets;
    size_t part_floats;
    long long q_stride, out_stride;   // elements
    int type, batch, group, chunks, window;   // chunks: groups of NT * 8 query heads per KV head
    float scale_log2;
};

template <int D, int NT, int KV>
struct Shape {
    static constexpr int kBytes = KV == NNC_E4M3 ? 1 : 2;
    static constexpr int kRow = D * kBytes;                  // bytes of a row
    static constexpr int kPB = kRow == 256 ? 16 : 32;        // positions of a warp's block
    static constexpr int kSub = kPB / 16;
    static constexpr int kTile = kWarps * kPB;
    static constexpr int kData = 2 * kPB * kRow;             // K rows, then V rows
    static constexpr int kStage = kData + (KV == NNC_E4M3 ? 2 * kPB : 0);   // then K scales, V scales
    static constexpr int kStages = kData == 8192 ? 3 : 5;
    static constexpr int kTilesD = D / 16;                   // 16-row tiles of O^T
    static constexpr int kOwn = kTilesD / kWarps;            // tiles that a warp merges
    static constexpr int kComb = kWarps * 3 * kOwn * 4 * 32 * 4;   // bytes: the pieces that warps hand to one another
    static constexpr int kSmem = kWarps * kStages * kStage + kComb;
    static constexpr int kSlotFloats = NT * (kTilesD * 128 + 16);   // a partial result: O^T fragments, (m, l) of 8 heads
};

struct AttnShared {
    float ml[kWarps][8][2];
    int sums[kWarps];
    int first_b, first_rest, is_last;
};

// byte offset of 16-byte piece c of row r, arranged so that eight rows of one column of pieces lie in different banks
template <int ROW> __device__ __forceinline__ int swizzled(int r, int c) {
    if constexpr (ROW >= 128) return r * ROW + ((c ^ (r & 7)) << 4);
    else return (r >> 1) * 128 + ((((r & 1) << 2 | c) ^ ((r >> 1) & 7)) << 4);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {
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
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}

// transposes an 8x8 matrix of 16-bit elements held one row per 4 lanes
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
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

// what a sequence attends to: positions [start, end), and its tiles, counted from `start` rounded down to 16
struct Reach {
    int start, end, tiles;
};
template <int TILE> __device__ __forceinline__ Reach reach_of(const PagedAttnParams &p, int b) {
    const int most = p.c.pages_per_seq << p.c.page_shift;
    int len = p.lens[b];
    len = max(0, min(len, most));
    Reach r;
    r.end = len;
    r.start = (p.window > 0 && len > p.window) ? len - p.window : 0;
    r.tiles = (len - (r.start & ~15) + TILE - 1) / TILE;
    return r;
}

// a place in the list of tiles
struct Place {
    Reach r;
    int b, hh, tile;   // hh: KV head * chunks + chunk of its query heads
};
template <int TILE> __device__ __forceinline__ void step(const PagedAttnParams &p, Place &at, int heads) {
    if (++at.tile < at.r.tiles) return;
    at.tile = 0;
    if (++at.hh < heads) return;
    at.hh = 0;
    do {
        if (++at.b >= p.batch) { at.r = Reach{0, 0, 0}; return; }   // past the list's end: nothing is taken from here
        at.r = reach_of<TILE>(p, at.b);
    } while (at.r.tiles == 0);
}

__device__ __forceinline__ void store_out(const PagedAttnParams &p, long long at, float v) {
    if (p.type == NNC_F32) reinterpret_cast<float *>(p.out)[at] = v;
    else if (p.type == NNC_BF16) reinterpret_cast<uint16_t *>(p.out)[at] = f32_to_bf16_bits(v);
    else reinterpret_cast<__half *>(p.out)[at] = __float2half_rn(v);
}

// QT, PT: terms of the queries and of the probabilities
template <int D, int NT, int KV, int QT, int PT>
__global__ void __launch_bounds__(kWarps * 32, 2) attn_paged_kernel(const PagedAttnParams p) {
    typedef Shape<D, NT, KV> S;
    constexpr bool BF = KV == NNC_BF16, CODES = KV == NNC_E4M3;
    constexpr int PB = S::kPB, TILE = S::kTile, ROW = S::kRow;
    // fp16 probabilities are scaled by 2^14, so that small ones keep their bits (the sums are scaled alike)
    constexpr float kLift = BF ? 0.f : 14.f;
    extern __shared__ __align__(128) char smem[];
    __shared__ AttnShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g8 = lane >> 2, t4 = lane & 3;
    const int heads = p.c.n_kv * p.chunks;

    // ---- the list: how many tiles there are, and where this CTA's share begins ----
    const int per = (p.batch + kWarps * 32 - 1) / (kWarps * 32);
    const int b_lo = min(tid * per, p.batch), b_hi = min(b_lo + per, p.batch);
    int mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += reach_of<TILE>(p, b).tiles;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sh.sums[warp] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { if (w < warp) before += sh.sums[w]; all += sh.sums[w]; }
    const int excl = before + incl - mine;
    const long long total = (long long)all * heads;   // the host bounds it by 2^31
    const int n_ctas = (int)min((long long)gridDim.x, total);
    const int cta = blockIdx.x;

    // sequences with nothing to attend to: zeros; and lengths that do not fit are reported
    for (int b = cta; b < p.batch; b += gridDim.x) {
        if (tid == 0 && p.lens[b] > (p.c.pages_per_seq << p.c.page_shift)) paged_complain(p.c);
        if (reach_of<TILE>(p, b).tiles) continue;
        const int n_q = p.c.n_kv * p.group;
        for (int i = tid; i < n_q * D; i += kWarps * 32) store_out(p, b * p.out_stride + i, 0.f);
        if (p.lse) for (int i = tid; i < n_q; i += kWarps * 32) p.lse[(long long)b * n_q + i] = -INFINITY;
    }
    if (cta >= n_ctas) return;
    const int t0 = (int)(total * cta / n_ctas), t1 = (int)(total * (cta + 1) / n_ctas);

    if (mine > 0) {
        const long long lo = (long long)excl * heads, hi = (long long)(excl + mine) * heads;
        if (t0 >= lo && t0 < hi) {
            long long rest = t0 - lo;
            int b = b_lo;
            for (; b < b_hi; ++b) {
                const long long n = (long long)reach_of<TILE>(p, b).tiles * heads;
                if (rest < n) break;
                rest -= n;
            }
            sh.first_b = b;
            sh.first_rest = (int)rest;
        }
    }
    __syncthreads();
    Place ahead;   // where the copies are
    ahead.b = sh.first_b;
    ahead.r = reach_of<TILE>(p, ahead.b);
    ahead.hh = sh.first_rest / ahead.r.tiles;
    ahead.tile = sh.first_rest - ahead.hh * ahead.r.tiles;
    Place now = ahead;   // where the products are

    // ---- copies of this warp's block of a tile ----
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S::kStages * S::kStage);
    int pages[S::kSub];
    auto find_pages = [&]() {   // one step before they are needed
        const int p0 = (ahead.r.start & ~15) + ahead.tile * TILE + warp * PB;
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
            pages[u] = -1;
            if (p0 + 16 * u < ahead.r.end)
                pages[u] = __ldg(p.c.table + (long long)ahead.b * p.c.pages_per_seq + ((p0 + 16 * u) >> p.c.page_shift));
        }
    };
    uint32_t present = 0;   // a bit per 16 positions of each stage: its page exists
    auto request = [&](int stage) {
        constexpr int kPieces = ROW / 16, kRowsPerStep = 32 / kPieces;
        const int p0 = (ahead.r.start & ~15) + ahead.tile * TILE + warp * PB;
        const int r0 = lane / kPieces, c0 = lane % kPieces, head = ahead.hh / p.chunks;
        const uint32_t base = ring + stage * S::kStage;
        present &= ~(((1u << S::kSub) - 1u) << (stage * S::kSub));
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
            const int pb = p0 + 16 * u;
            if (pb >= ahead.r.end) break;
            const bool there = (unsigned)pages[u] < (unsigned)p.c.n_pages;
            if (there) present |= 1u << (stage * S::kSub + u);
            else if (lane == 0) paged_complain(p.c);
            const long long row = there ? paged_row(p.c, pages[u], head, pb & ((1 << p.c.page_shift) - 1)) : 0;
            const char *ks = p.c.k + row * ROW + r0 * ROW + c0 * 16, *vs = p.c.v + row * ROW + r0 * ROW + c0 * 16;
#pragma unroll
            for (int i = 0; i < 16 / kRowsPerStep; ++i) {
                const int r = r0 + i * kRowsPerStep;
                const bool live = there && pb + r >= ahead.r.start && pb + r < ahead.r.end;
                const int dst = swizzled<ROW>(16 * u + r, c0);
                copy16(base + dst, live ? ks + i * kRowsPerStep * ROW : p.c.k, live);
                copy16(base + PB * ROW + dst, live ? vs + i * kRowsPerStep * ROW : p.c.v, live);
            }
            if constexpr (CODES) {
                if (lane < 2)
                    copy16(base + S::kData + lane * PB + 16 * u, there ? (lane ? p.c.v_scale : p.c.k_scale) + row : p.c.k_scale, there);
            }
        }
    };

    const int n = t1 - t0;
    find_pages();
    int asked = 0;
#pragma unroll
    for (int st = 0; st < S::kStages - 1; ++st) {
        if (asked < n) {
            request(st);
            ++asked;
            step<TILE>(p, ahead, heads);
            if (asked < n) find_pages();
        }
        copy_commit();
    }

    // ---- per (sequence, head) state ----
    uint32_t qf[NT][QT][D / 16][2];
    float qmul[NT][2];
    float o[NT][S::kTilesD][4], m_run[NT][2], l_run[NT][2];
    int piece_first = 0;   // list index of the piece's first tile, in this CTA's share

    auto begin_piece = [&]() {
        const int kv_head = now.hh / p.chunks, chunk = now.hh - kv_head * p.chunks;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // queries: lane (g8, t4) holds head g8's elements of contraction columns 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9 of
            // every step of 16; with codes, a key's four neighbouring codes 4 t4 .. 4 t4 + 3 stand in those columns
            const int g = chunk * (8 * NT) + nt * 8 + g8;
            const bool there = g < p.group;
            const long long at = now.b * p.q_stride + (long long)(kv_head * p.group + (there ? g : 0)) * D;
            float f[D / 16][4];
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const int ia = CODES ? 16 * s + 4 * t4 : 16 * s + 2 * t4, ib = CODES ? ia + 2 : ia + 8;
                if (p.type == NNC_F32) {
                    const float2 a = *reinterpret_cast<const float2 *>(p.q + (at + ia) * 4), b = *reinterpret_cast<const float2 *>(p.q + (at + ib) * 4);
                    f[s][0] = a.x; f[s][1] = a.y; f[s][2] = b.x; f[s][3] = b.y;
                } else {
                    const uint32_t a = *reinterpret_cast<const uint32_t *>(p.q + (at + ia) * 2), b = *reinterpret_cast<const uint32_t *>(p.q + (at + ib) * 2);
                    if (p.type == NNC_BF16) { f[s][0] = bf16_lo(a); f[s][1] = bf16_hi(a); f[s][2] = bf16_lo(b); f[s][3] = bf16_hi(b); }
                    else {
                        f[s][0] = __half2float(__ushort_as_half((uint16_t)a)); f[s][1] = __half2float(__ushort_as_half((uint16_t)(a >> 16)));
                        f[s][2] = __half2float(__ushort_as_half((uint16_t)b)); f[s][3] = __half2float(__ushort_as_half((uint16_t)(b >> 16)));
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) { if (!there) f[s][e] = 0.f; top = fmaxf(top, fabsf(f[s][e])); }
            }
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
                m_run[nt][e] = -INFINITY;
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

    // lane's row and piece in the four 8x8 matrices of an ldmatrix: K (rows = positions) and V (transposed)
    const int lr = lane & 7, lm = lane >> 3;
    auto products = [&](int stage) {
        const int p0 = (now.r.start & ~15) + now.tile * TILE + warp * PB;
        if (p0 >= now.r.end) return;
        const uint32_t kb = ring + stage * S::kStage, vb = kb + PB * ROW;
        const char *scales = smem + warp * (S::kStages * S::kStage) + stage * S::kStage + S::kData;
        float s[S::kSub][NT][4], ev[S::kSub][2];
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][0] = s[u][nt][1] = s[u][nt][2] = s[u][nt][3] = 0.f;
            if constexpr (!CODES) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t a[4];
                    ldsm4(a, kb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, 2 * c + (lm >> 1)));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < QT; ++i) mma16816<BF>(s[u][nt], a[0], a[1], a[2], a[3], qf[nt][i][c]);
                }
            } else {
#pragma unroll
                for (int c = 0; c < D / 16; c += 2) {
                    uint32_t a[4];
                    ldsm4(a, kb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, c + (lm >> 1)));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t a0 = e4m3x2_to_f16x2(a[2 * e] & 0xffffu), a2 = e4m3x2_to_f16x2(a[2 * e] >> 16);
                        const uint32_t a1 = e4m3x2_to_f16x2(a[2 * e + 1] & 0xffffu), a3 = e4m3x2_to_f16x2(a[2 * e + 1] >> 16);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < QT; ++i) mma16816<false>(s[u][nt], a0, a1, a2, a3, qf[nt][i][c + e]);
                    }
                }
            }
            const bool there = present >> (stage * S::kSub + u) & 1u;
#pragma unroll
            for (int r = 0; r < 2; ++r) {   // rows g8 and g8 + 8
                const int pos = p0 + 16 * u + g8 + 8 * r;
                const bool live = there && pos >= now.r.start && pos < now.r.end;
                float ks = 1.f;
                ev[u][r] = 0.f;
                if constexpr (CODES) {
                    const int at = 16 * u + g8 + 8 * r;
                    const uint32_t bk = live ? (uint8_t)scales[at] : 127u, bv = live ? (uint8_t)scales[PB + at] : 127u;
                    ks = scale_from_byte(bk);
                    ev[u][r] = (float)((int)bv - 127);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float x = s[u][nt][2 * r + e] * qmul[nt][e] * ks + ev[u][r];
                        s[u][nt][2 * r + e] = live ? x : -INFINITY;
                    }
            }
        }
        // ---- online softmax; with codes, of the scores plus the value rows' exponents ----
        uint32_t pf[S::kSub][NT][PT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float alpha[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mx = -INFINITY;
#pragma unroll
                for (int u = 0; u < S::kSub; ++u) mx = fmaxf(mx, fmaxf(s[u][nt][e], s[u][nt][2 + e]));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                const float m_new = fmaxf(m_run[nt][e], mx);
                const float ref = (m_new == -INFINITY ? 0.f : m_new) - kLift;   // nothing attended so far: every weight is 0
                alpha[e] = exp2f(m_run[nt][e] - kLift - ref);
                m_run[nt][e] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < S::kSub; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float w = exp2f(s[u][nt][2 * r + e] - ref);
                        s[u][nt][2 * r + e] = w;
                        sum += CODES ? w * __uint_as_float((uint32_t)(127 - (int)ev[u][r]) << 23) : w;
                    }
                l_run[nt][e] = l_run[nt][e] * alpha[e] + sum;
            }
            if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int i = 0; i < S::kTilesD; ++i) { o[nt][i][0] *= alpha[0]; o[nt][i][1] *= alpha[1]; o[nt][i][2] *= alpha[0]; o[nt][i][3] *= alpha[1]; }
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
        //      with codes 16 i + 2 g8 and 16 i + 2 g8 + 1 ----
#pragma unroll
        for (int u = 0; u < S::kSub; ++u) {
            if (p0 + 16 * u >= now.r.end) break;   // nothing was copied there: what the stage holds may be no number
            if constexpr (!CODES) {
#pragma unroll
                for (int i = 0; i < S::kTilesD; ++i) {
                    uint32_t a[4];
                    ldsm4_trans(a, vb + swizzled<ROW>(16 * u + lr + (lm >> 1) * 8, 2 * i + (lm & 1)));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < PT; ++j) mma16816<BF>(o[nt][i], a[0], a[1], a[2], a[3], pf[u][nt][j]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < S::kTilesD; i += 2) {
                    uint32_t a[4];   // positions 0-7 and 8-15 of piece i, then of piece i + 1
                    ldsm4_trans(a, vb + swizzled<ROW>(16 * u + lr + (lm & 1) * 8, i + (lm >> 1)));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // a lane holds two neighbouring codes of two positions: pair them by code
                        const uint32_t x = __byte_perm(a[2 * e], 0, 0x3120), y = __byte_perm(a[2 * e + 1], 0, 0x3120);
                        const uint32_t a0 = e4m3x2_to_f16x2(x & 0xffffu), a1 = e4m3x2_to_f16x2(x >> 16);
                        const uint32_t a2 = e4m3x2_to_f16x2(y & 0xffffu), a3 = e4m3x2_to_f16x2(y >> 16);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int j = 0; j < PT; ++j) mma16816<false>(o[nt][i + e], a0, a1, a2, a3, pf[u][nt][j]);
                    }
                }
            }
        }
    };

    // ---- writing results: o_own, M, L hold this warp's tiles of the joined result ----
    auto write_head_tiles = [&](int nt, const float (&own)[S::kOwn][4], const float (&M)[2], const float (&L)[2]) {
        const int kv_head = now.hh / p.chunks, chunk = now.hh - kv_head * p.chunks;
        const int n_q = p.c.n_kv * p.group;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int g = chunk * (8 * NT) + nt * 8 + 2 * t4 + e;
            if (g >= p.group) continue;
            const float inv = L[e] == 0.f ? 0.f : 1.f / L[e];
            const long long at = now.b * p.out_stride + (long long)(kv_head * p.group + g) * D;
#pragma unroll
            for (int j = 0; j < S::kOwn; ++j) {
                const int i = warp * S::kOwn + j;
                const int d0 = CODES ? 16 * i + 2 * g8 : 16 * i + g8, d1 = CODES ? d0 + 1 : d0 + 8;
                store_out(p, at + d0, own[j][e] * inv);
                store_out(p, at + d1, own[j][2 + e] * inv);
            }
            if (p.lse && warp == 0 && g8 == 0)
                p.lse[(long long)now.b * n_q + kv_head * p.group + g] =
                    L[e] == 0.f ? -INFINITY : (M[e] + log2f(L[e])) * 0.69314718055994530942f;
        }
    };

    float (*comb)[3][S::kOwn][32][4] = reinterpret_cast<float (*)[3][S::kOwn][32][4]>(smem + kWarps * S::kStages * S::kStage);

    auto end_piece = [&](int last_index) {   // list indices, counted from the list's begin
        const int item_lo = last_index - now.tile, item_hi = item_lo + now.r.tiles;   // this (sequence, head)'s tiles
        const int first = t0 + piece_first;
        const bool whole = first == item_lo && last_index + 1 == item_hi;
        // partial results: slot 0 of a CTA for a piece that continues an earlier CTA's, slot 1 for one that starts here
        float *slot = p.part + (size_t)(2 * cta + (first == item_lo ? 1 : 0)) * S::kSlotFloats;
        if (!whole && !NNC_BC((size_t)(2 * cta + 2) * S::kSlotFloats <= p.part_floats, 3201)) return;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = l_run[nt][e];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                if (g8 == 0) { sh.ml[warp][2 * t4 + e][0] = m_run[nt][e] == -INFINITY ? -INFINITY : m_run[nt][e] - kLift; sh.ml[warp][2 * t4 + e][1] = l; }
            }
            float own[S::kOwn][4];
#pragma unroll
            for (int i = 0; i < S::kTilesD; ++i) {
                const int to = i / S::kOwn, j = i % S::kOwn;
                const float4 v = make_float4(o[nt][i][0], o[nt][i][1], o[nt][i][2], o[nt][i][3]);
                if (to == warp) { own[j][0] = v.x; own[j][1] = v.y; own[j][2] = v.z; own[j][3] = v.w; }
                else *reinterpret_cast<float4 *>(comb[to][warp < to ? warp : warp - 1][j][lane]) = v;
            }
            __syncthreads();
            float M[2], L[2], wgt[kWarps][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                M[e] = -INFINITY;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) M[e] = fmaxf(M[e], sh.ml[w][2 * t4 + e][0]);
                const float ref = M[e] == -INFINITY ? 0.f : M[e];
                L[e] = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    wgt[w][e] = exp2f(sh.ml[w][2 * t4 + e][0] - ref);
                    L[e] = fmaf(wgt[w][e], sh.ml[w][2 * t4 + e][1], L[e]);
                }
            }
            float sum[S::kOwn][4];
#pragma unroll
            for (int j = 0; j < S::kOwn; ++j) sum[j][0] = sum[j][1] = sum[j][2] = sum[j][3] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
#pragma unroll
                for (int j = 0; j < S::kOwn; ++j) {
                    float4 v = make_float4(own[j][0], own[j][1], own[j][2], own[j][3]);
                    if (w != warp) v = *reinterpret_cast<const float4 *>(comb[warp][w < warp ? w : w - 1][j][lane]);
                    sum[j][0] = fmaf(wgt[w][0], v.x, sum[j][0]); sum[j][1] = fmaf(wgt[w][1], v.y, sum[j][1]);
                    sum[j][2] = fmaf(wgt[w][0], v.z, sum[j][2]); sum[j][3] = fmaf(wgt[w][1], v.w, sum[j][3]);
                }
            if (whole) {
                write_head_tiles(nt, sum, M, L);
            } else {
                float *o_part = slot + nt * (S::kTilesD * 128 + 16);
#pragma unroll
                for (int j = 0; j < S::kOwn; ++j)
                    *reinterpret_cast<float4 *>(o_part + ((warp * S::kOwn + j) * 32 + lane) * 4) = make_float4(sum[j][0], sum[j][1], sum[j][2], sum[j][3]);
                if (warp == 0 && g8 == 0)
                    *reinterpret_cast<float4 *>(o_part + S::kTilesD * 128 + 4 * t4) = make_float4(M[0], L[0], M[1], L[1]);
            }
            __syncthreads();
        }
        if (whole) return;
        // ---- the CTAs of this (sequence, head): the one that finishes last joins the pieces, in order ----
        const int c_lo = (int)(((item_lo + 1ll) * n_ctas - 1) / total), c_hi = (int)(((long long)item_hi * n_ctas - 1) / total);
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            const int last = atomicAdd(&p.tickets[c_lo], 1u) == (unsigned)(c_hi - c_lo);
            if (last) p.tickets[c_lo] = 0u;
            sh.is_last = last;
        }
        __syncthreads();
        if (!sh.is_last) return;
        __threadfence();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            auto piece = [&](int c) {   // the first piece lies in its CTA's slot 1, the others in slot 0
                return p.part + (size_t)(2 * c + (c == c_lo ? 1 : 0)) * S::kSlotFloats + nt * (S::kTilesD * 128 + 16);
            };
            float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f};
            for (int c = c_lo + g8; c <= c_hi; c += 8) {
                const float4 ml = __ldcg(reinterpret_cast<const float4 *>(piece(c) + S::kTilesD * 128 + 4 * t4));
                M[0] = fmaxf(M[0], ml.x); M[1] = fmaxf(M[1], ml.z);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                M[e] = fmaxf(M[e], __shfl_xor_sync(0xffffffffu, M[e], 4));
                M[e] = fmaxf(M[e], __shfl_xor_sync(0xffffffffu, M[e], 8));
                M[e] = fmaxf(M[e], __shfl_xor_sync(0xffffffffu, M[e], 16));
            }
            const float ref0 = M[0] == -INFINITY ? 0.f : M[0], ref1 = M[1] == -INFINITY ? 0.f : M[1];
            float sum[S::kOwn][4];
#pragma unroll
            for (int j = 0; j < S::kOwn; ++j) sum[j][0] = sum[j][1] = sum[j][2] = sum[j][3] = 0.f;
#pragma unroll 4
            for (int c = c_lo; c <= c_hi; ++c) {
                const float *pc = piece(c);
                const float4 ml = __ldcg(reinterpret_cast<const float4 *>(pc + S::kTilesD * 128 + 4 * t4));
                const float w0 = exp2f(ml.x - ref0), w1 = exp2f(ml.z - ref1);
                L[0] = fmaf(w0, ml.y, L[0]); L[1] = fmaf(w1, ml.w, L[1]);
#pragma unroll
                for (int j = 0; j < S::kOwn; ++j) {
                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(pc + ((warp * S::kOwn + j) * 32 + lane) * 4));
                    sum[j][0] = fmaf(w0, v.x, sum[j][0]); sum[j][1] = fmaf(w1, v.y, sum[j][1]);
                    sum[j][2] = fmaf(w0, v.z, sum[j][2]); sum[j][3] = fmaf(w1, v.w, sum[j][3]);
                }
            }
            write_head_tiles(nt, sum, M, L);
        }
    };

    begin_piece();
    for (int it = 0, stage = 0; it < n; ++it) {
        copy_wait<S::kStages - 2>();
        __syncwarp();
        const int refill = stage == 0 ? S::kStages - 1 : stage - 1;   // the stage that the step before this one used
        if (asked < n) {
            request(refill);
            ++asked;
            step<TILE>(p, ahead, heads);
            if (asked < n) find_pages();
        }
        copy_commit();
        products(stage);
        __syncwarp();
        const bool ends = it + 1 == n || now.tile + 1 == now.r.tiles;
        if (ends) end_piece(t0 + it);
        if (it + 1 < n) {
            step<TILE>(p, now, heads);
            if (ends) { piece_first = it + 1; begin_piece(); }
        }
        stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }
    copy_wait<0>();
}

template <int D, int NT, int KV, int QT, int PT>
cudaError_t launch_one(const LaunchCtx &lc, const PagedAttnParams &p) {
    typedef Shape<D, NT, KV> S;
    static unsigned long long raised = 0;
    auto kern = attn_paged_kernel<D, NT, KV, QT, PT>;
    cudaError_t e = ensure_dynamic_smem(kern, S::kSmem, &raised);
    if (e != cudaSuccess) return e;
    const long long most = ((long long)p.c.pages_per_seq << p.c.page_shift);
    const long long tiles = ((most + 15 + S::kTile - 1) / S::kTile) * p.batch * p.c.n_kv * p.chunks;   // the longest list the table allows
    if (tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    long long ctas = 2ll * lc.sm_count;
    if (ctas > kPagedMaxCtas) ctas = kPagedMaxCtas;
    const long long fit = (long long)(p.part_floats / (2 * S::kSlotFloats));
    if (ctas > fit) ctas = fit;
    if (ctas > tiles) ctas = tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = lc.stream;
    if (lc.launches) ++*lc.launches;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

// 16-bit results: queries as one exact term, probabilities as two; fp32 results: as many terms as fp32 has bits for
template <int D, int NT>
cudaError_t launch_typed(const LaunchCtx &lc, const PagedAttnParams &p, int kv) {
    const bool f32 = p.type == NNC_F32;
    if (kv == NNC_BF16) return f32 ? launch_one<D, NT, NNC_BF16, 3, 3>(lc, p) : launch_one<D, NT, NNC_BF16, 1, 2>(lc, p);
    if (kv == NNC_F16) return f32 ? launch_one<D, NT, NNC_F16, 2, 2>(lc, p) : launch_one<D, NT, NNC_F16, 1, 2>(lc, p);
    return f32 ? launch_one<D, NT, NNC_E4M3, 2, 2>(lc, p) : launch_one<D, NT, NNC_E4M3, 1, 2>(lc, p);
}

}  // namespace

cudaError_t launch_attn_paged(const LaunchCtx &lc, const void *q, const nnc_paged_kv &cache, const int32_t *lens, void *out, float *lse,
                              int type, int batch, int n_q_heads, int64_t q_stride, int64_t out_stride, float scale, int window,
                              void *scratch, size_t scratch_bytes) {
    PagedAttnParams p;
    p.c = paged_view(cache, lc.status);
    p.q = (const char *)q; p.out = (char *)out; p.lse = lse; p.lens = lens;
    p.tickets = (uint32_t *)scratch;
    p.part = (float *)((char *)scratch + NNC_ATTN_PAGED_TICKET_BYTES);
    p.part_floats = (scratch_bytes - NNC_ATTN_PAGED_TICKET_BYTES) / 4;
    p.q_stride = q_stride; p.out_stride = out_stride;
    p.type = type; p.batch = batch; p.window = window;
    p.group = n_q_heads / cache.n_kv_heads;
    p.scale_log2 = scale * 1.4426950408889634f;
    const bool two = p.group > 8;   // one 8-column operand, or two, that share every key and value fragment
    p.chunks = two ? (p.group + 15) / 16 : 1;
    if (cache.head_dim == 64) return two ? launch_typed<64, 2>(lc, p, cache.type) : launch_typed<64, 1>(lc, p, cache.type);
    return two ? launch_typed<128, 2>(lc, p, cache.type) : launch_typed<128, 1>(lc, p, cache.type);
}

}  // namespace nnc
