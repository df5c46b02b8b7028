// Rows of the paged key-value cache: written (rounded to 16 bits, or quantised to E4M3 codes with a power-of-two scale per
// row) and read back.
//
// Bound by the rows' bytes on both sides.  head_dim / 8 neighbouring lanes own the key row and the value row of one (token,
// KV head): eight elements each, so a 16-bit row moves as 16-byte vectors and a row of codes as 8-byte ones, and a row's
// largest magnitude is found by shuffles among its lanes, with the row read once.  The key row's and the value row's loads
// are in flight together.
#include <cuda_fp16.h>

#include "paged.cuh"

namespace nnc {

namespace {

struct RowsParams {
    PagedView c;
    char *k, *v;
    const int32_t *pos, *seq;
    long long row_stride, head_stride;   // bytes
    int n_tokens;
};

constexpr int kScaleMax = 60;   // a row's exponent lies in [-60, 60]

template <int TYPE> struct Vec8 { uint4 q[TYPE == NNC_F32 ? 2 : 1]; };   // eight elements of a 16-bit type or of fp32

template <int TYPE> __device__ __forceinline__ Vec8<TYPE> load8(const char *p) {
    Vec8<TYPE> r;
    if constexpr (TYPE == NNC_F32) {   // the second vector finds the first one's sectors in L1
        r.q[0] = reinterpret_cast<const uint4 *>(p)[0];
        r.q[1] = reinterpret_cast<const uint4 *>(p)[1];
    } else {
        r.q[0] = __ldcg(reinterpret_cast<const uint4 *>(p));   // used once
    }
    return r;
}
template <int TYPE> __device__ __forceinline__ void store8(char *p, const Vec8<TYPE> &r) {
    reinterpret_cast<uint4 *>(p)[0] = r.q[0];
    if constexpr (TYPE == NNC_F32) reinterpret_cast<uint4 *>(p)[1] = r.q[1];
}

template <int TYPE> __device__ __forceinline__ void unpack8(const Vec8<TYPE> &r, float (&f)[8]) {
    if constexpr (TYPE == NNC_F32) {
        const uint32_t w[8] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    } else {
        const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == NNC_BF16) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
            else {
                f[2 * i] = __half2float(__ushort_as_half((uint16_t)w[i]));
                f[2 * i + 1] = __half2float(__ushort_as_half((uint16_t)(w[i] >> 16)));
            }
        }
    }
}
template <int TYPE> __device__ __forceinline__ Vec8<TYPE> pack8(const float (&f)[8]) {
    Vec8<TYPE> r;
    if constexpr (TYPE == NNC_F32) {
        r.q[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        r.q[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == NNC_BF16) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
            else
                w[i] = (uint32_t)__half_as_ushort(__float2half_rn(f[2 * i])) |
                       (uint32_t)__half_as_ushort(__float2half_rn(f[2 * i + 1])) << 16;
        }
        r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}

// Largest finite magnitudes, as fp32 bits (they order like the values), of a key row and a value row that LANES neighbouring
// lanes hold eight elements each of.  16-bit types: two elements at a time, and the two rows together through the shuffles;
// the maxima pass over NaN, and a row with an infinity is looked through again without it.
template <int TYPE, int LANES>
__device__ __forceinline__ void tops_of(const Vec8<TYPE> &k, const Vec8<TYPE> &v, const float (&fk)[8], const float (&fv)[8], uint32_t &top_k,
                                        uint32_t &top_v) {
    constexpr uint32_t kInf = 0x7f800000u;
    if constexpr (TYPE == NNC_F32) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) { a = fmaxf(a, fabsf(fk[i])); b = fmaxf(b, fabsf(fv[i])); }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
            b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, o));
        }
        top_k = __float_as_uint(a);
        top_v = __float_as_uint(b);
    } else {
        auto max2 = [](uint32_t a, uint32_t b) {
            uint32_t r;
            if constexpr (TYPE == NNC_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        };
        constexpr uint32_t kAbs = 0x7fff7fffu;
        const uint32_t a = max2(max2(k.q[0].x & kAbs, k.q[0].y & kAbs), max2(k.q[0].z & kAbs, k.q[0].w & kAbs));
        const uint32_t b = max2(max2(v.q[0].x & kAbs, v.q[0].y & kAbs), max2(v.q[0].z & kAbs, v.q[0].w & kAbs));
        uint32_t m = max2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));   // low half: keys, high half: values
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) m = max2(m, __shfl_xor_sync(0xffffffffu, m, o));
        const Vec8<TYPE> both{{make_uint4(m, 0u, 0u, 0u)}};
        float f[8];
        unpack8<TYPE>(both, f);
        top_k = __float_as_uint(f[0]);
        top_v = __float_as_uint(f[1]);
    }
    if (__any_sync(0xffffffffu, top_k == kInf || top_v == kInf)) {
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = __float_as_uint(fk[i]) & 0x7fffffffu, y = __float_as_uint(fv[i]) & 0x7fffffffu;
            if (x < kInf && x > a) a = x;
            if (y < kInf && y > b) b = y;
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
            a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
            b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
        }
        top_k = a;
        top_v = b;
    }
    if (top_k > kInf) top_k = 0;   // nothing but NaN
    if (top_v > kInf) top_v = 0;
}

// Codes of eight values of a row with the given largest magnitude, and the row's exponent, biased by 127.
__device__ __forceinline__ uint2 quantise8(const float (&f)[8], uint32_t top, uint32_t &byte) {
    // top = 1.m * 2^E = (1.m / 1.75) * 448 * 2^(E - 8): e = E - 8, one more where 1.m is over 1.75
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
    e = top == 0u ? 0 : max(-kScaleMax, min(kScaleMax, e));
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);   // exact: the codes do not depend on how x / 2^e is formed
    byte = (uint32_t)(e + 127);
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t pair;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(pair) : "f"(f[2 * i + 1] * down), "f"(f[2 * i] * down));
        c[i] = pair;
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

__device__ __forceinline__ void dequantise8(const uint2 codes, uint32_t byte, float (&f)[8]) {
    const float up = scale_from_byte(byte);
    const uint32_t w[4] = {codes.x & 0xffffu, codes.x >> 16, codes.y & 0xffffu, codes.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t h = e4m3x2_to_f16x2(w[i]);
        f[2 * i] = __half2float(__ushort_as_half((uint16_t)h)) * up;
        f[2 * i + 1] = __half2float(__ushort_as_half((uint16_t)(h >> 16))) * up;
    }
}

// D: head_dim; KV: the cache's type; TYPE: the type of the rows outside; R: rows a thread takes part in, whose loads are in
// flight together
template <int D, int KV, int TYPE, bool WRITE, int R>
__global__ void __launch_bounds__(256) kv_rows_kernel(const RowsParams p) {
    constexpr int kLanes = D / 8, kRows = 256 / kLanes;   // rows a CTA takes at once
    constexpr int kOutside = TYPE == NNC_F32 ? 32 : 16;   // bytes of a lane's eight elements outside the cache
    const int lane = threadIdx.x % kLanes;
    pdl_launch_dependents();
    pdl_wait();
    const unsigned rows = (unsigned)p.n_tokens * (unsigned)p.c.n_kv;
    const unsigned row0 = blockIdx.x * (unsigned)(kRows * R) + threadIdx.x / kLanes;
    int s[R], n[R], h[R], page[R];
    bool live[R];
    long long off[R], at[R];
    Vec8<TYPE> k[R], v[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const unsigned row = row0 + i * kRows;
        live[i] = row < rows;
        const unsigned t = live[i] ? row / (unsigned)p.c.n_kv : 0u;
        h[i] = live[i] ? (int)(row - t * p.c.n_kv) : 0;
        s[i] = p.seq ? p.seq[t] : (int)t;
        n[i] = p.pos[t];
        off[i] = t * p.row_stride + h[i] * p.head_stride + lane * kOutside;
        if constexpr (WRITE) { k[i] = load8<TYPE>(p.k + off[i]); v[i] = load8<TYPE>(p.v + off[i]); }
    }
    // the addresses: padding is left out, what lies outside is left out and reported
#pragma unroll
    for (int i = 0; i < R; ++i) {
        live[i] = live[i] && s[i] >= 0 && n[i] >= 0;
        const int column = n[i] >> p.c.page_shift;
        page[i] = -1;
        if (live[i] && s[i] < p.c.n_seqs && column < p.c.pages_per_seq) page[i] = p.c.table[(long long)s[i] * p.c.pages_per_seq + column];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (live[i] && (unsigned)page[i] >= (unsigned)p.c.n_pages) {
            live[i] = false;
            if (lane == 0 && h[i] == 0) paged_complain(p.c);
        }
        at[i] = live[i] ? paged_row(p.c, page[i], h[i], n[i] & ((1 << p.c.page_shift) - 1)) : 0;
        live[i] = live[i] && NNC_BC(at[i] >= 0 && at[i] < paged_rows(p.c) && h[i] < p.c.n_kv, 3301);
    }
    if constexpr (WRITE) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long b = at[i] * (2 * D) + lane * 16;
            if constexpr (KV == TYPE) {
                if (!live[i]) continue;
                store8<TYPE>(p.c.k + b, k[i]);
                store8<TYPE>(p.c.v + b, v[i]);
            } else {
                float fk[8], fv[8];
                unpack8<TYPE>(k[i], fk);
                unpack8<TYPE>(v[i], fv);
                if constexpr (KV == NNC_E4M3) {
                    uint32_t top_k, top_v, ke, ve;   // every lane of the warp takes part in the shuffles, whether its row is live or not
                    tops_of<TYPE, kLanes>(k[i], v[i], fk, fv, top_k, top_v);
                    const uint2 kc = quantise8(fk, top_k, ke), vc = quantise8(fv, top_v, ve);
                    if (!live[i]) continue;
                    *reinterpret_cast<uint2 *>(p.c.k + at[i] * D + lane * 8) = kc;
                    *reinterpret_cast<uint2 *>(p.c.v + at[i] * D + lane * 8) = vc;
                    if (lane == 0) { p.c.k_scale[at[i]] = (uint8_t)ke; p.c.v_scale[at[i]] = (uint8_t)ve; }
                } else {
                    if (!live[i]) continue;
                    store8<KV>(p.c.k + b, pack8<KV>(fk));
                    store8<KV>(p.c.v + b, pack8<KV>(fv));
                }
            }
        }
    } else {
        // a row that is not there is read from the pool's first one and not stored
        if constexpr (KV == NNC_E4M3) {
            uint2 kc[R], vc[R];
            uint32_t ke[R], ve[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                kc[i] = __ldcg(reinterpret_cast<const uint2 *>(p.c.k + at[i] * D + lane * 8));
                vc[i] = __ldcg(reinterpret_cast<const uint2 *>(p.c.v + at[i] * D + lane * 8));
                ke[i] = p.c.k_scale[at[i]];
                ve[i] = p.c.v_scale[at[i]];
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float fk[8], fv[8];
                dequantise8(kc[i], ke[i], fk);
                dequantise8(vc[i], ve[i], fv);
                k[i] = pack8<TYPE>(fk);
                v[i] = pack8<TYPE>(fv);
            }
        } else {
            Vec8<KV> ck[R], cv[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long long b = at[i] * (2 * D) + lane * 16;
                ck[i] = load8<KV>(p.c.k + b);
                cv[i] = load8<KV>(p.c.v + b);
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if constexpr (KV == TYPE) { k[i] = ck[i]; v[i] = cv[i]; }
                else {
                    float fk[8], fv[8];
                    unpack8<KV>(ck[i], fk);
                    unpack8<KV>(cv[i], fv);
                    k[i] = pack8<TYPE>(fk);
                    v[i] = pack8<TYPE>(fv);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!live[i]) continue;
            store8<TYPE>(p.k + off[i], k[i]);
            store8<TYPE>(p.v + off[i], v[i]);
        }
    }
}

template <int D, int KV, int TYPE, bool WRITE>
cudaError_t launch_sized(const LaunchCtx &lc, const RowsParams &p) {
    constexpr int kRows = 256 / (D / 8);
    const long long rows = (long long)p.n_tokens * p.c.n_kv;
    const long long once = (rows + kRows - 1) / kRows;
    LaunchCtx early = lc;
    early.pdl = true;   // the kernel waits for its predecessor itself
    // Two rows a thread where that still leaves every SM several CTAs; otherwise one, for the shortest way through.  Reading
    // 63315 rows of 8 heads x 128 codes: 40 us with one, 33.7 with two, 34.2 with three, 34.6 with four
    if (once >= 16ll * lc.sm_count)
        return launch(early, kv_rows_kernel<D, KV, TYPE, WRITE, 2>, dim3((unsigned)((once + 1) / 2)), dim3(256), p);
    return launch(early, kv_rows_kernel<D, KV, TYPE, WRITE, 1>, dim3((unsigned)once), dim3(256), p);
}

template <int D, int KV>
cudaError_t launch_rows(const LaunchCtx &lc, const RowsParams &p, bool write, int type) {
    switch (type) {
        case NNC_F32: return write ? launch_sized<D, KV, NNC_F32, true>(lc, p) : launch_sized<D, KV, NNC_F32, false>(lc, p);
        case NNC_BF16: return write ? launch_sized<D, KV, NNC_BF16, true>(lc, p) : launch_sized<D, KV, NNC_BF16, false>(lc, p);
        default: return write ? launch_sized<D, KV, NNC_F16, true>(lc, p) : launch_sized<D, KV, NNC_F16, false>(lc, p);
    }
}

}  // namespace

cudaError_t launch_kv_paged(const LaunchCtx &lc, const nnc_paged_kv &cache, bool write, void *k, void *v, int type, int n_tokens,
                            int64_t row_stride, int64_t head_stride, const int32_t *pos, const int32_t *seq) {
    const int el = type == NNC_F32 ? 4 : 2;
    RowsParams p;
    p.c = paged_view(cache, lc.status);
    p.k = (char *)k; p.v = (char *)v; p.pos = pos; p.seq = seq;
    p.row_stride = row_stride * el; p.head_stride = head_stride * el;
    p.n_tokens = n_tokens;
    if (cache.head_dim == 64) {
        if (cache.type == NNC_BF16) return launch_rows<64, NNC_BF16>(lc, p, write, type);
        if (cache.type == NNC_F16) return launch_rows<64, NNC_F16>(lc, p, write, type);
        return launch_rows<64, NNC_E4M3>(lc, p, write, type);
    }
    if (cache.type == NNC_BF16) return launch_rows<128, NNC_BF16>(lc, p, write, type);
    if (cache.type == NNC_F16) return launch_rows<128, NNC_F16>(lc, p, write, type);
    return launch_rows<128, NNC_E4M3>(lc, p, write, type);
}

}  // namespace nnc
