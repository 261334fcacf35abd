// A pool of pages as kernels see it (include/cacheroute.h), for those that keep pages (cr_pages.cu) and those that write
// and read what is in them (cr_kv.cu).
#pragma once

#include "cr_internal.cuh"

struct pages_in {
    uint8_t *cache;
    int32_t *ref, *table, *lens;
    uint32_t layers, n_pages, page, page_log2, kv_heads, head_dim, n_seqs, max_pages;
    uint32_t size_log2;  // bytes of an element: 1 << size_log2
    uint64_t layer_stride, kv_stride, page_stride, token_stride, head_stride;  // elements
    float *scale;        // 8 bits: [layers][2][n_pages][kv_heads][page / block], else NULL
    uint32_t block_log2;
    uint32_t *status;
    // Layer l2 / 2, keys (l2 even) or values.
    __device__ __forceinline__ uint8_t *plane(uint32_t l2) const
    {
        return cache + (((uint64_t)(l2 >> 1) * layer_stride + (uint64_t)(l2 & 1) * kv_stride) << size_log2);
    }
    // Scales of a page in that plane, [kv_heads][page / block].
    __device__ __forceinline__ float *scales(uint32_t l2, uint32_t p) const
    {
        return scale + (((uint64_t)l2 * n_pages + p) * kv_heads << (page_log2 - block_log2));
    }
};

static inline pages_in cr_pages_input(cr_ctx *ctx, const cr_kv_pages *pg)
{
    pages_in P = {};
    P.cache = static_cast<uint8_t *>(pg->d_cache);
    P.ref = pg->d_ref;
    P.table = pg->d_table;
    P.lens = pg->d_lens;
    P.layers = pg->layers;
    P.n_pages = pg->n_pages;
    P.page = pg->page;
    while ((1u << P.page_log2) < pg->page) ++P.page_log2;
    P.kv_heads = pg->kv_heads;
    P.head_dim = pg->head_dim;
    P.n_seqs = pg->n_seqs;
    P.max_pages = pg->max_pages;
    P.layer_stride = pg->layer_stride;
    P.kv_stride = pg->kv_stride;
    P.page_stride = pg->page_stride;
    P.token_stride = pg->token_stride;
    P.head_stride = pg->head_stride;
    P.status = ctx->d_status;
    P.size_log2 = 1;
    if (cr_in_8bit(pg->dtype)) {
        P.size_log2 = 0;
        P.scale = pg->d_scale;
        while ((1u << P.block_log2) < pg->block) ++P.block_log2;
    }
    return P;
}

// Limits of a pool (cr_pages.cu).
int cr_pages_check(cr_ctx *ctx, const char *who, const cr_kv_pages *pg);
// Writes new tokens' keys and values, rotated or not (cr_kv.cu).
int cr_append(cr_ctx *ctx, const char *who, const cr_kv_pages *pg, uint32_t layer, const cr_rotary *rotary, const cr_append_args *args);
