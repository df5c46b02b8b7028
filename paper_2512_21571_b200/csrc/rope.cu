// Rotary positions on rows of heads: y = R(position * freq) x on the first rotary_dim elements of every head.
//
// Bound by reading x and writing y.  The angles depend on the token and the pair only, so a CTA works out the cosines and
// sines of its tokens once, in shared memory, and all heads use them.  A thread owns up to eight pairs of one head (two 16-byte
// loads and stores of 16-bit values) in several tokens, whose loads are on their way while the angles are worked out.  The
// angle is position * freq as a sum of two doubles, reduced to an eighth of a turn before it is rounded to fp32: what is left then is
// off by at most 2^-28 turns, however far the position (one double would be off by 2^-24 at 2^31; 8192 x 40 x 128: 28.6 and 28.7 us).
#include <cuda_fp16.h>

#include "common.cuh"
#include "nnc_internal.h"

namespace nnc {

namespace {

struct RopeParams {
    const char *x;
    char *y;
    const int32_t *pos;
    const double *freq;
    long long x_row, x_head, y_row, y_head;   // elements
    int n_tokens, n_heads, head_dim, rot, tokens_per_cta, units;   // units: work items per head
    int abreast;                                         // vector form: tokens that a CTA's threads take at once
    float amplitude;
    bool inverse;
};

// tokens whose loads a thread has in flight when there are many
template <int TYPE> constexpr int kMany = TYPE == NNC_F32 ? 2 : 3;

// N neighbouring elements
template <int TYPE, int N> struct Piece {
    static constexpr int kWords = N * (TYPE == NNC_F32 ? 4 : 2) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                // 16-bit values are used once; the second vector of fp32 values finds the first one's sectors in L1
                const uint4 v = kWords == 4 ? __ldcg(reinterpret_cast<const uint4 *>(p)) : reinterpret_cast<const uint4 *>(p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (kWords == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x; w[1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        }
    }
    __device__ __forceinline__ void store(char *p) const {
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else if constexpr (kWords == 2) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else {
            *reinterpret_cast<uint32_t *>(p) = w[0];
        }
    }
    __device__ __forceinline__ void get(float (&f)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (TYPE == NNC_F32) f[i] = __uint_as_float(w[i]);
            else if constexpr (TYPE == NNC_BF16) f[i] = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
            else f[i] = __half2float(__ushort_as_half((uint16_t)(w[i / 2] >> (16 * (i & 1)))));
        }
    }
    __device__ __forceinline__ void put(const float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (TYPE == NNC_F32) w[i] = __float_as_uint(f[i]);
            else if constexpr (TYPE == NNC_BF16) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
            else {
                const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
};

template <int TYPE> struct Scalar {
    typedef uint16_t raw;
    static __device__ __forceinline__ float get(raw r) {
        if constexpr (TYPE == NNC_BF16) return bf16_bits_to_f32(r);
        else return __half2float(__ushort_as_half(r));
    }
    static __device__ __forceinline__ raw put(float f) {
        if constexpr (TYPE == NNC_BF16) return f32_to_bf16_bits(f);
        else return __half_as_ushort(__float2half_rn(f));
    }
};
template <> struct Scalar<NNC_F32> {
    typedef float raw;
    static __device__ __forceinline__ float get(float f) { return f; }
    static __device__ __forceinline__ float put(float f) { return f; }
};

// cosine and sine of pos * freq, times the amplitude.  The angle in turns is a sum of two doubles, so that the far position's whole turns
// take nothing from the fraction: both products' rounding errors (from fused multiply-adds) and the rest of 1 / 2 pi are in the second one.
__device__ __forceinline__ float2 turn_of(int pos, double freq, float amplitude, bool inverse) {
    constexpr double kTurn = 0.15915494309189533576888376337251, kTurnRest = -9.839338337591243e-18;   // 1 / 2 pi = the double + the rest
    const double angle = (double)pos * freq, angle_rest = fma((double)pos, freq, -angle);
    const double turns = angle * kTurn, turns_rest = fma(angle, kTurn, -turns) + fma(angle, kTurnRest, angle_rest * kTurn);
    const double quarters = rint(turns * 4.0);
    const float f = (float)((turns - quarters * 0.25) + turns_rest);   // within an eighth of a turn; the difference is exact
    float s, c;
    sincospif(2.f * f, &s, &c);
    const int q = (int)((long long)quarters & 3);
    if (q & 1) { const float t = c; c = -s; s = t; }
    if (q & 2) { c = -c; s = -s; }
    if (inverse) s = -s;
    return make_float2(c * amplitude, s * amplitude);
}

// Vector form: a unit is N pairs (or, past the rotated part, N elements that only pass through).  Thread: one unit of one head
// (more, if a token has more units than the CTA has threads), in M tokens.
template <int TYPE, bool INTERLEAVED, int N, int M>
__global__ void __launch_bounds__(512) rope_kernel(const RopeParams p) {
    constexpr int el = TYPE == NNC_F32 ? 4 : 2;
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ float4 turn[];   // [tokens_per_cta][N / 2][rot / 2N]: two pairs each; lanes of one head read side by side
    const int half = p.rot / 2, rot_units = half / N;
    const int t0 = blockIdx.x * p.tokens_per_cta, tokens = min(p.tokens_per_cta, p.n_tokens - t0);
    const int per_token = p.n_heads * p.units;
    const int first = threadIdx.x / per_token;                       // the thread's first token; past it, every abreast-th
    const int each = p.abreast > 1 ? per_token : (int)blockDim.x;    // units that the CTA's threads cover of a token
    Piece<TYPE, N> a[M], b[M];
    long long x_at = 0, y_at = 0;
    int u = 0, at_a = 0, at_b = 0;
    auto load = [&](int r) {
        const int h = r / p.units;
        u = r - h * p.units;
        if (u >= rot_units) at_a = at_b = p.rot + N * (u - rot_units);
        else if (INTERLEAVED) { at_a = 2 * N * u; at_b = at_a + N; }
        else { at_a = N * u; at_b = half + N * u; }
        x_at = (long long)(t0 + first) * p.x_row + h * p.x_head;
        y_at = (long long)(t0 + first) * p.y_row + h * p.y_head;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (first + m * p.abreast >= tokens) break;
            if (!NNC_BC(h < p.n_heads && at_a >= 0 && at_a + N <= p.head_dim && at_b + N <= p.head_dim && t0 + first + m * p.abreast < p.n_tokens, 3401)) break;
            const char *x = p.x + (x_at + (long long)(m * p.abreast) * p.x_row) * el;
            a[m].load(x + at_a * el);
            if (u < rot_units) b[m].load(x + at_b * el);
        }
    };
    int r = threadIdx.x - first * per_token;
    const bool in = first < p.abreast && r < per_token;   // (a token wider than the CTA: first is 0)
    if (in) load(r);
    for (int k = threadIdx.x; k < tokens * half; k += blockDim.x) {
        const int t = k / half, i = k - t * half;
        reinterpret_cast<float2 *>(turn)[((t * (N / 2) + i % N / 2) * rot_units + i / N) * 2 + (i & 1)] =
            turn_of(p.pos[t0 + t], p.freq[i], p.amplitude, p.inverse);
    }
    __syncthreads();
    if (!in) return;
    for (;;) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int t = first + m * p.abreast;
            if (t >= tokens || !NNC_BC(t < p.tokens_per_cta && at_b + N <= p.head_dim, 3402)) break;
            char *y = p.y + (y_at + (long long)(m * p.abreast) * p.y_row) * el;
            if (u < rot_units) {
                float fa[N], fb[N];
                a[m].get(fa);
                b[m].get(fb);
#pragma unroll
                for (int q = 0; q < N / 2; ++q) {
                    const float4 cs = turn[(t * (N / 2) + q) * rot_units + u];   // pairs 2q and 2q + 1
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int j = 2 * q + e;
                        float &xa = INTERLEAVED ? (j < N / 2 ? fa[2 * j % N] : fb[2 * j % N]) : fa[j];
                        float &xb = INTERLEAVED ? (j < N / 2 ? fa[2 * j % N + 1] : fb[2 * j % N + 1]) : fb[j];
                        const float c = e ? cs.z : cs.x, s = e ? cs.w : cs.y, va = xa, vb = xb;
                        xa = va * c - vb * s;
                        xb = vb * c + va * s;
                    }
                }
                a[m].put(fa);
                b[m].put(fb);
                b[m].store(y + at_b * el);
            }
            a[m].store(y + at_a * el);
        }
        r += each;
        if (r >= per_token) break;
        load(r);
    }
}

// Element by element, for sizes and strides that do not allow vectors: a unit is one pair, or one element that passes through.
template <int TYPE, bool INTERLEAVED>
__global__ void __launch_bounds__(512) rope_plain_kernel(const RopeParams p) {
    typedef Scalar<TYPE> E;
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ float4 turn4[];
    float2 *turn = reinterpret_cast<float2 *>(turn4);   // [tokens_per_cta][rot / 2]
    const int half = p.rot / 2;
    const int t0 = blockIdx.x * p.tokens_per_cta, tokens = min(p.tokens_per_cta, p.n_tokens - t0);
    const int per_token = p.n_heads * p.units;
    for (int k = threadIdx.x; k < tokens * half; k += blockDim.x) {
        const int t = k / half;
        turn[k] = turn_of(p.pos[t0 + t], p.freq[k - t * half], p.amplitude, p.inverse);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * per_token; i += blockDim.x) {
        const int t = i / per_token, r = i - t * per_token, h = r / p.units, u = r - h * p.units;
        if (!NNC_BC(h < p.n_heads && (u < half || p.rot + u - half < p.head_dim) && t0 + t < p.n_tokens, 3403)) continue;
        const typename E::raw *x = reinterpret_cast<const typename E::raw *>(p.x) + (long long)(t0 + t) * p.x_row + h * p.x_head;
        typename E::raw *y = reinterpret_cast<typename E::raw *>(p.y) + (long long)(t0 + t) * p.y_row + h * p.y_head;
        if (u >= half) {
            y[p.rot + u - half] = x[p.rot + u - half];
            continue;
        }
        const int ia = INTERLEAVED ? 2 * u : u, ib = INTERLEAVED ? 2 * u + 1 : half + u;
        const float2 cs = turn[t * half + u];
        const float xa = E::get(x[ia]), xb = E::get(x[ib]);
        y[ia] = E::put(xa * cs.x - xb * cs.y);
        y[ib] = E::put(xb * cs.x + xa * cs.y);
    }
}

template <int TYPE, int N>
cudaError_t launch_sized(const LaunchCtx &lc, const RopeParams &p, bool many, bool interleaved, dim3 grid, dim3 block, int smem) {
    constexpr int M = kMany<TYPE>;
    LaunchCtx early = lc;
    early.pdl = true;   // the kernels wait for their predecessor themselves
    if constexpr (N == 1) return launch_smem(early, interleaved ? rope_plain_kernel<TYPE, true> : rope_plain_kernel<TYPE, false>, grid, block, (size_t)smem, p);
    else
        return launch_smem(early, many ? (interleaved ? rope_kernel<TYPE, true, N, M> : rope_kernel<TYPE, false, N, M>)
                                       : (interleaved ? rope_kernel<TYPE, true, N, 1> : rope_kernel<TYPE, false, N, 1>), grid, block, (size_t)smem, p);
}

template <int TYPE>
cudaError_t launch_typed(const LaunchCtx &lc, const RopeParams &p, int n, bool many, bool interleaved, dim3 grid, dim3 block, int smem) {
    switch (n) {
        case 8: return launch_sized<TYPE, 8>(lc, p, many, interleaved, grid, block, smem);
        case 4: return launch_sized<TYPE, 4>(lc, p, many, interleaved, grid, block, smem);
        case 2: return launch_sized<TYPE, 2>(lc, p, many, interleaved, grid, block, smem);
        default: return launch_sized<TYPE, 1>(lc, p, many, interleaved, grid, block, smem);
    }
}

}  // namespace

cudaError_t launch_rope(const LaunchCtx &lc, const void *x, void *y, int type, int n_tokens, int n_heads, int head_dim, int64_t x_row,
                        int64_t x_head, int64_t y_row, int64_t y_head, const int32_t *positions, const double *freq,
                        int rotary_dim, bool interleaved, bool inverse, float amplitude) {
    const int el = type == NNC_F32 ? 4 : 2, half = rotary_dim / 2;
    RopeParams p;
    p.x = (const char *)x; p.y = (char *)y; p.pos = positions; p.freq = freq;
    p.x_row = x_row; p.x_head = x_head; p.y_row = y_row; p.y_head = y_head;
    p.n_tokens = n_tokens; p.n_heads = n_heads; p.head_dim = head_dim; p.rot = rotary_dim;
    p.amplitude = amplitude; p.inverse = inverse;
    const bool copy_rest = x != y && rotary_dim < head_dim;
    // the largest piece of n elements that pairs, what passes through, pointers and strides are all whole multiples of (16-byte
    // vectors at most).  8192 x 40 heads of 80 bf16: 20 of them turned 57 us with n = 2, 40 turned 38 with n = 4; 99 and 88 with n = 1
    int n = 8;
    for (; n > 1; n /= 2) {
        const int bytes = n * el < 16 ? n * el : 16;
        bool fits = half % n == 0 && head_dim % n == 0 && !(((uintptr_t)x | (uintptr_t)y) % bytes);
        for (int64_t s : {x_row, x_head, y_row, y_head}) fits = fits && (s * el) % bytes == 0;
        if (fits) break;
    }
    p.units = half / n;
    if (copy_rest) p.units += (head_dim - rotary_dim) / n;
    const long long per_token = (long long)n_heads * p.units;
    // A CTA's threads take one token abreast where that gives them 128 units or more, and else as many as give 256.  With enough
    // tokens for several CTAs per SM a thread has kMany of them in flight; otherwise one, for the shortest way through.
    const int m = type == NNC_F32 ? kMany<NNC_F32> : kMany<NNC_BF16>;
    long long abreast = per_token >= 128 ? 1 : 256 / per_token;
    if (abreast * m * half > 4096) abreast = 4096 / (m * half) > 1 ? 4096 / (m * half) : 1;   // 32 KB of angles at most
    long long threads = abreast * per_token;
    if (threads > 512) threads = 512;
    p.abreast = (int)abreast;
    const bool many = n > 1 && n_tokens >= 4ll * abreast * m * lc.sm_count;
    long long tokens = abreast * (many ? m : 1);
    p.tokens_per_cta = (int)tokens;
    const dim3 grid((unsigned)((n_tokens + tokens - 1) / tokens)), block((unsigned)((threads + 31) / 32 * 32));
    const int smem = (int)(tokens * half * sizeof(float2));
    switch (type) {
        case NNC_F32: return launch_typed<NNC_F32>(lc, p, n, many, interleaved, grid, block, smem);
        case NNC_BF16: return launch_typed<NNC_BF16>(lc, p, n, many, interleaved, grid, block, smem);
        default: return launch_typed<NNC_F16>(lc, p, n, many, interleaved, grid, block, smem);
    }
}

}  // namespace nnc
