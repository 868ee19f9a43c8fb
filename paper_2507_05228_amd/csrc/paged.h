// Shared by the operators of the paged cache (host side).
#pragma once
#include "common.h"

// log2 of the page size
static inline int page_shift(const cascade_paged_cache *c) { return __builtin_ctz((unsigned)c->page_size); }

// The limits of the descriptor, for every entry point that takes one
static inline int32_t check_paged_cache(const cascade_paged_cache *c) {
    if (!c || !c->k_pages || !c->v_pages || !c->page_table || !c->kv_len || !c->page_refs) return CASCADE_EINVAL;
    if (c->n_layers <= 0 || c->n_pages <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || c->n_seqs <= 0 ||
        c->n_shards <= 0 || c->max_pages <= 0)
        return CASCADE_EINVAL;
    if (c->dtype != CASCADE_F32 && c->dtype != CASCADE_BF16) return CASCADE_EUNSUPPORTED;
    if (c->head_dim > 256 || c->head_dim % (c->dtype == CASCADE_BF16 ? 8 : 4)) return CASCADE_EUNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return CASCADE_EUNSUPPORTED;
    // rows of the pool, rows of a list and entries of the lists count in 32 bits, those of a list with a step of 64 keys behind them,
    // entries with a round of 4096 sequences
    if (c->n_shards > 1024 || c->n_kv_heads > 65535 || (int64_t)c->n_pages * c->page_size > INT32_MAX ||
        (int64_t)c->max_pages * c->page_size > INT32_MAX - 64 || (int64_t)c->n_seqs * c->n_shards * c->max_pages > INT32_MAX - 4096)
        return CASCADE_EUNSUPPORTED;
    // steps of 32 rows over all lists of a sequence, too
    if ((int64_t)c->n_shards * c->max_pages * c->page_size > ((int64_t)1 << 35)) return CASCADE_EUNSUPPORTED;
    if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages) % 16) return CASCADE_EUNSUPPORTED;
    return CASCADE_OK;
}

// Elements of one layer's pool of keys (or values)
static inline int64_t layer_elems(const cascade_paged_cache *c) {
    return (int64_t)c->n_pages * c->n_kv_heads * c->page_size * c->head_dim;
}
