// What the kernels over a paged cache share (pages.cu, chunk_attention*.cu).
#pragma once
#include <cuda_fp16.h>
#include "device_helpers.cuh"

struct PagePool {
    unsigned char *kc, *vc;
    void *ks, *kz, *vs, *vz;                         // float32, or binary16 in the M16 instances
    long long page_stride, head_stride;              // in tokens
    int n_pages, page_tokens;
};
inline PagePool page_pool_of(const squat_page_pool *p)
{
    return {p->k_codes, p->v_codes, p->k_scales, p->k_zeros, p->v_scales, p->v_zeros, p->page_stride, p->head_stride, p->n_pages, p->page_tokens};
}
// Token index of the place that `slot` names in head h (in the pool's strides).
__device__ __forceinline__ long long token_at_slot(const PagePool &pool, int slot, int h)
{
    const int page = slot / pool.page_tokens;
    return (long long)page * pool.page_stride + (long long)h * pool.head_stride + (slot - page * pool.page_tokens);
}
