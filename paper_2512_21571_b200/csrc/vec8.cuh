// Eight elements of fp32, bf16 or fp16 as 16-byte vectors, and as fp32 numbers.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "nnc_internal.h"

namespace nnc {

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

}  // namespace nnc
