// Check of a radix_cache (host arithmetic) and the view that the kernels take of it.
#pragma once
#include "common.h"
#include "kernels.h"

static inline int cache_shape(const radix_cache* c, CacheView* v) {
    if (!c) return RADIX_ERR_NULL_POINTER;
    if (c->n_layers <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->n_pages <= 0 || c->max_seqs <= 0 || c->max_pages <= 0)
        return RADIX_ERR_BAD_SIZE;
    if (c->dtype != RADIX_F32 && c->dtype != RADIX_BF16 && c->dtype != RADIX_F16) return RADIX_ERR_UNSUPPORTED;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
        return RADIX_ERR_UNSUPPORTED;
    // the head sizes that a forward has in the type
    if (c->dtype == RADIX_F32 ? (c->head_dim % 4 != 0 || c->head_dim > 128) : c->head_dim != 128) return RADIX_ERR_UNSUPPORTED;
    if (c->n_kv_heads > 65535 || c->n_layers > 65535) return RADIX_ERR_UNSUPPORTED;
    if ((int64_t)c->max_pages * c->page_size > INT32_MAX) return RADIX_ERR_BAD_SIZE;          // positions are 32-bit
    if (c->n_pages > (1 << 28) || c->max_seqs > RADIX_CACHE_MAX_SLOTS) return RADIX_ERR_UNSUPPORTED;
    int shift = 4;
    while ((1 << shift) < c->page_size) ++shift;
    *v = {(char*)c->pages, c->page_refs, c->page_table, c->seq_lens, c->n_layers, c->n_pages, c->n_kv_heads, c->head_dim, c->page_size,
          shift, c->max_seqs, c->max_pages, 0, 0, 0};
    v->piece_bytes = (size_t)c->page_size * c->head_dim * (c->dtype == RADIX_F32 ? 4 : 2);
    v->page_bytes = 2 * (size_t)c->n_kv_heads * v->piece_bytes;
    if (v->page_bytes > INT32_MAX) return RADIX_ERR_UNSUPPORTED;
    v->layer_bytes = (size_t)c->n_pages * v->page_bytes;                                      // below 2^59
    if (v->layer_bytes > (size_t)INT64_MAX / (size_t)c->n_layers) return RADIX_ERR_UNSUPPORTED;
    return RADIX_OK;
}

static inline int cache_view(const radix_cache* c, CacheView* v) {
    const int rc = cache_shape(c, v);
    if (rc != RADIX_OK) return rc;
    if (!c->pages || !c->page_refs || !c->page_table || !c->seq_lens) return RADIX_ERR_NULL_POINTER;
    if (((uintptr_t)c->pages & 15) != 0) return RADIX_ERR_MISALIGNED;
    return RADIX_OK;
}
