// Device-side view of a paged key-value cache (nnc_paged_kv) and the address and scale arithmetic its kernels share.
#pragma once
#include "common.cuh"
#include "nnc_internal.h"

namespace nnc {

struct PagedView {
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t *table;
    int *status;
    int n_pages, page_shift, n_kv, n_seqs, pages_per_seq;
};

inline PagedView paged_view(const nnc_paged_kv &c, int *status) {
    PagedView p;
    p.k = (char *)c.k; p.v = (char *)c.v;
    p.k_scale = c.k_scale; p.v_scale = c.v_scale;
    p.table = c.page_table;
    p.status = status;
    p.n_pages = c.n_pages;
    p.page_shift = __builtin_ctz((unsigned)c.page_size);
    p.n_kv = c.n_kv_heads; p.n_seqs = c.n_seqs; p.pages_per_seq = c.pages_per_seq;
    return p;
}

__device__ __forceinline__ void paged_complain(const PagedView &c) {
    if (c.status) atomicOr(c.status, NNC_STATUS_PAGED_ADDRESS);
}

// row (of one KV head, counted over the pool) of position `slot` of `page`; 64 bits, a pool may hold more than 2^31 rows
__device__ __forceinline__ long long paged_row(const PagedView &c, int page, int head, int slot) {
    return (((long long)page * c.n_kv + head) << c.page_shift) + slot;
}

// rows of the pool
__device__ __forceinline__ long long paged_rows(const PagedView &c) { return ((long long)c.n_pages * c.n_kv) << c.page_shift; }

// 2^(byte - 127): a row's scale (byte 0 is 2^-127, a subnormal; 255 stands for no number)
__device__ __forceinline__ float scale_from_byte(uint32_t byte) {
    return byte == 0u ? __uint_as_float(0x00400000u) : byte == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte << 23);
}

// two E4M3 codes (low byte first) as an fp16 pair; every code is exactly an fp16 value
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
    uint32_t r;
    asm("{ .reg .b16 t; cvt.u16.u32 t, %1; cvt.rn.f16x2.e4m3x2 %0, t; }" : "=r"(r) : "r"(codes));
    return r;
}

}  // namespace nnc
