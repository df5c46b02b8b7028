// Rotary positions on rows of heads: y = R(position * freq) x on the first rotary_dim elements of every head.
//
// Bound by reading x and writing y.  The angles depend on the token and the pair only, so a CTA works out the cosines and
// sines of its tokens once, in shared memory, and all heads use them; a thread owns eight pairs of one head (two 16-byte
// loads and stores of 16-bit values) that it requests before the angles are known.  The angle is position * freq in 64 bits,
// reduced to an eighth of a turn before it is rounded to fp32: what is left then is off by at most 2^-28 turns, however far
// the position.
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
    float amplitude;
    bool inverse, copy_rest;
};

template <int TYPE> struct Elem { typedef uint16_t raw; };
template <> struct Elem<NNC_F32> { typedef float raw; };

template <int TYPE> __device__ __forceinline__ float to_f32(typename Elem<TYPE>::raw r) {
    if constexpr (TYPE == NNC_F32) return r;
    else if constexpr (TYPE == NNC_BF16) return bf16_bits_to_f32(r);
    else return __half2float(__ushort_as_half(r));
}
template <int TYPE> __device__ __forceinline__ typename Elem<TYPE>::raw from_f32(float f) {
    if constexpr (TYPE == NNC_F32) return f;
    else if constexpr (TYPE == NNC_BF16) return f32_to_bf16_bits(f);
    else return __half_as_ushort(__float2half_rn(f));
}

// cosine and sine of pos * freq, times the amplitude
__device__ __forceinline__ float2 turn_of(int pos, double freq, float amplitude, bool inverse) {
    const double turns = (double)pos * freq * 0.15915494309189533576888376337251;
    const double quarters = rint(turns * 4.0);
    const float f = (float)(turns - quarters * 0.25);   // exact difference, within an eighth of a turn; then one rounding
    float s, c;
    sincospif(2.f * f, &s, &c);
    const int q = (int)((long long)quarters & 3);
    if (q & 1) { const float t = c; c = -s; s = t; }
    if (q & 2) { c = -c; s = -s; }
    if (inverse) s = -s;
    return make_float2(c * amplitude, s * amplitude);
}

template <int TYPE>
struct alignas(16) Eight { typename Elem<TYPE>::raw e[8]; };

// VEC: a unit is eight pairs, moved as 16-byte vectors (or eight elements that only pass through); otherwise it is one pair
// (or one element), for sizes and strides that do not allow vectors.
template <int TYPE, bool VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(512) rope_kernel(const RopeParams p) {
    typedef typename Elem<TYPE>::raw raw;
    extern __shared__ float2 turn[];   // [tokens_per_cta][rot / 2]
    const int half = p.rot / 2;
    const int t0 = blockIdx.x * p.tokens_per_cta;
    const int tokens = min(p.tokens_per_cta, p.n_tokens - t0);
    const int rot_units = VEC ? half / 8 : half;
    const int per_token = p.n_heads * p.units, items = tokens * per_token;
    for (int i = threadIdx.x; i < tokens * half; i += blockDim.x) {
        const int t = i / half;
        turn[i] = turn_of(p.pos[t0 + t], p.freq[i - t * half], p.amplitude, p.inverse);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < items; i += blockDim.x) {
        const int t = i / per_token, r = i - t * per_token, h = r / p.units, u = r - h * p.units;
        const raw *x = reinterpret_cast<const raw *>(p.x) + (t0 + t) * p.x_row + h * p.x_head;
        raw *y = reinterpret_cast<raw *>(p.y) + (t0 + t) * p.y_row + h * p.y_head;
        if (u >= rot_units) {   // elements past the rotated part
            if constexpr (VEC) {
                const int at = p.rot + 8 * (u - rot_units);
                *reinterpret_cast<Eight<TYPE> *>(y + at) = *reinterpret_cast<const Eight<TYPE> *>(x + at);
            } else {
                const int at = p.rot + (u - rot_units);
                y[at] = x[at];
            }
            continue;
        }
        const float2 *cs = turn + t * half + (VEC ? 8 * u : u);
        if constexpr (VEC) {
            const int a0 = INTERLEAVED ? 16 * u : 8 * u, b0 = INTERLEAVED ? 16 * u + 8 : half + 8 * u;
            Eight<TYPE> a = *reinterpret_cast<const Eight<TYPE> *>(x + a0), b = *reinterpret_cast<const Eight<TYPE> *>(x + b0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                raw &ea = INTERLEAVED ? (j < 4 ? a.e[2 * j & 7] : b.e[2 * j & 7]) : a.e[j];
                raw &eb = INTERLEAVED ? (j < 4 ? a.e[(2 * j & 7) + 1] : b.e[(2 * j & 7) + 1]) : b.e[j];
                const float xa = to_f32<TYPE>(ea), xb = to_f32<TYPE>(eb);
                ea = from_f32<TYPE>(xa * cs[j].x - xb * cs[j].y);
                eb = from_f32<TYPE>(xb * cs[j].x + xa * cs[j].y);
            }
            *reinterpret_cast<Eight<TYPE> *>(y + a0) = a;
            *reinterpret_cast<Eight<TYPE> *>(y + b0) = b;
        } else {
            const int ia = INTERLEAVED ? 2 * u : u, ib = INTERLEAVED ? 2 * u + 1 : half + u;
            const float xa = to_f32<TYPE>(x[ia]), xb = to_f32<TYPE>(x[ib]);
            y[ia] = from_f32<TYPE>(xa * cs->x - xb * cs->y);
            y[ib] = from_f32<TYPE>(xb * cs->x + xa * cs->y);
        }
    }
}

template <int TYPE>
cudaError_t launch_typed(const LaunchCtx &lc, const RopeParams &p, bool vec, bool interleaved, dim3 grid, dim3 block, int smem) {
    auto kern = vec ? (interleaved ? rope_kernel<TYPE, true, true> : rope_kernel<TYPE, true, false>)
                    : (interleaved ? rope_kernel<TYPE, false, true> : rope_kernel<TYPE, false, false>);
    if (lc.launches) ++*lc.launches;
    kern<<<grid, block, smem, lc.stream>>>(p);
    return cudaGetLastError();
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
    p.copy_rest = x != y && rotary_dim < head_dim;
    // vectors need whole groups of eight pairs, whole 16-byte pieces of what passes through, and 16-byte rows and heads
    bool vec = half % 8 == 0 && head_dim % 8 == 0 && !(((uintptr_t)x | (uintptr_t)y) & 15);
    for (int64_t s : {x_row, x_head, y_row, y_head}) vec = vec && (s * el) % 16 == 0;
    p.units = vec ? half / 8 : half;
    if (p.copy_rest) p.units += vec ? (head_dim - rotary_dim) / 8 : head_dim - rotary_dim;
    const long long per_token = (long long)n_heads * p.units;
    // one token a CTA where a token fills one, as many as give 256 items otherwise (the angles' table: 16 KB at most)
    long long tokens = per_token >= 256 ? 1 : 256 / per_token;
    if (tokens * half > 2048) tokens = half >= 2048 ? 1 : 2048 / half;
    if (tokens > n_tokens) tokens = n_tokens;
    p.tokens_per_cta = (int)tokens;
    long long threads = (tokens * per_token + 31) / 32 * 32;
    if (threads > 512) threads = 512;
    const dim3 grid((unsigned)((n_tokens + tokens - 1) / tokens)), block((unsigned)threads);
    const int smem = (int)(tokens * half * sizeof(float2));
    switch (type) {
        case NNC_F32: return launch_typed<NNC_F32>(lc, p, vec, interleaved, grid, block, smem);
        case NNC_BF16: return launch_typed<NNC_BF16>(lc, p, vec, interleaved, grid, block, smem);
        default: return launch_typed<NNC_F16>(lc, p, vec, interleaved, grid, block, smem);
    }
}

}  // namespace nnc
