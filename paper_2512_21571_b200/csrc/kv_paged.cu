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
    r.q[0] = reinterpret_cast<const uint4 *>(p)[0];
    if constexpr (TYPE == NNC_F32) r.q[1] = reinterpret_cast<const uint4 *>(p)[1];
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

// Eight values of a row whose `lanes` lanes hold the rest: the row's exponent (biased by 127) and these values' codes.
template <int LANES> __device__ __forceinline__ uint2 quantise8(const float (&f)[8], uint32_t &byte) {
    uint32_t top = 0;   // largest finite magnitude, as bits: they order like the values
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __float_as_uint(f[i]) & 0x7fffffffu;
        if (m < 0x7f800000u && m > top) top = m;
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
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

// D: head_dim; KV: the cache's type; TYPE: the type of the rows outside
template <int D, int KV, int TYPE, bool WRITE>
__global__ void __launch_bounds__(256) kv_rows_kernel(const RowsParams p) {
    constexpr int kLanes = D / 8, kRowsPerCta = 256 / kLanes;
    const int lane = threadIdx.x % kLanes;
    const long long row = (long long)blockIdx.x * kRowsPerCta + threadIdx.x / kLanes;
    const long long t_all = row / p.c.n_kv;
    const int h = (int)(row - t_all * p.c.n_kv);
    const bool in = t_all < p.n_tokens;
    const int t = in ? (int)t_all : 0;
    const int s = p.seq ? p.seq[t] : t, n = p.pos[t];
    constexpr int kOutside = TYPE == NNC_F32 ? 32 : 16;   // bytes of a lane's eight elements outside the cache
    const long long off = t * p.row_stride + h * p.head_stride + lane * kOutside;
    Vec8<TYPE> k, v;
    if constexpr (WRITE) { k = load8<TYPE>(p.k + off); v = load8<TYPE>(p.v + off); }
    // the address: padding is left out, what lies outside is left out and reported
    bool live = in && s >= 0 && n >= 0;
    long long at = 0;
    if (live) {
        const int column = n >> p.c.page_shift;
        int page = -1;
        if (s < p.c.n_seqs && column < p.c.pages_per_seq) page = p.c.table[(long long)s * p.c.pages_per_seq + column];
        if (page < 0 || page >= p.c.n_pages) {
            live = false;
            if (lane == 0 && h == 0) paged_complain(p.c);
        } else {
            at = paged_row(p.c, page, h, n & ((1 << p.c.page_shift) - 1));
        }
    }
    if constexpr (WRITE) {
        if constexpr (KV == TYPE) {
            if (!live) return;
            const long long b = at * (2 * D) + lane * 16;
            store8<TYPE>(p.c.k + b, k);
            store8<TYPE>(p.c.v + b, v);
        } else {
            float fk[8], fv[8];
            unpack8<TYPE>(k, fk);
            unpack8<TYPE>(v, fv);
            if constexpr (KV == NNC_E4M3) {
                uint32_t ke, ve;   // every lane of the warp takes part in the shuffles, whether its row is live or not
                const uint2 kc = quantise8<kLanes>(fk, ke), vc = quantise8<kLanes>(fv, ve);
                if (!live) return;
                *reinterpret_cast<uint2 *>(p.c.k + at * D + lane * 8) = kc;
                *reinterpret_cast<uint2 *>(p.c.v + at * D + lane * 8) = vc;
                if (lane == 0) { p.c.k_scale[at] = (uint8_t)ke; p.c.v_scale[at] = (uint8_t)ve; }
            } else {
                if (!live) return;
                const long long b = at * (2 * D) + lane * 16;
                store8<KV>(p.c.k + b, pack8<KV>(fk));
                store8<KV>(p.c.v + b, pack8<KV>(fv));
            }
        }
    } else {
        if (!live) return;
        if constexpr (KV == TYPE) {
            const long long b = at * (2 * D) + lane * 16;
            k = load8<TYPE>(p.c.k + b);
            v = load8<TYPE>(p.c.v + b);
        } else {
            float fk[8], fv[8];
            if constexpr (KV == NNC_E4M3) {
                const uint2 kc = *reinterpret_cast<const uint2 *>(p.c.k + at * D + lane * 8);
                const uint2 vc = *reinterpret_cast<const uint2 *>(p.c.v + at * D + lane * 8);
                dequantise8(kc, p.c.k_scale[at], fk);
                dequantise8(vc, p.c.v_scale[at], fv);
            } else {
                const long long b = at * (2 * D) + lane * 16;
                unpack8<KV>(load8<KV>(p.c.k + b), fk);
                unpack8<KV>(load8<KV>(p.c.v + b), fv);
            }
            k = pack8<TYPE>(fk);
            v = pack8<TYPE>(fv);
        }
        store8<TYPE>(p.k + off, k);
        store8<TYPE>(p.v + off, v);
    }
}

template <int D, int KV>
cudaError_t launch_rows(const LaunchCtx &lc, const RowsParams &p, bool write, int type) {
    const long long rows = (long long)p.n_tokens * p.c.n_kv;
    constexpr int kRowsPerCta = 256 / (D / 8);
    const dim3 grid((unsigned)((rows + kRowsPerCta - 1) / kRowsPerCta)), block(256);
#define NNC_ROWS_CASE(TT) \
    return write ? launch(lc, kv_rows_kernel<D, KV, TT, true>, grid, block, p) : launch(lc, kv_rows_kernel<D, KV, TT, false>, grid, block, p)
    switch (type) {
        case NNC_F32: NNC_ROWS_CASE(NNC_F32);
        case NNC_BF16: NNC_ROWS_CASE(NNC_BF16);
        default: NNC_ROWS_CASE(NNC_F16);
    }
#undef NNC_ROWS_CASE
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
