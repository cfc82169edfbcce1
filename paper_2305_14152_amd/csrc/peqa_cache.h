// The paged key-value cache on the device side: the descriptor as kernels take it, and the host's check of it.
#pragma once

#include "../../include/peqa.h"
#include "peqa_device.h"

namespace peqa {

// peqa_kv_cache with what kernels derive from it.
struct CacheArgs {
    void *k, *v;
    const int32_t *table;
    const float *k_scale, *v_scale;
    long long page_stride, head_stride, slot_stride, table_stride;
    int n_pages, page_shift, page_mask, kv_heads;
    int n_seqs, n_blocks;
};

inline CacheArgs cache_args(const peqa_kv_cache *C)
{
    CacheArgs a{};
    a.k = C->k; a.v = C->v; a.table = C->table;
    a.k_scale = C->k_scale; a.v_scale = C->v_scale;
    a.page_stride = C->page_stride; a.head_stride = C->head_stride; a.slot_stride = C->slot_stride;
    a.table_stride = C->table_stride;
    a.n_pages = C->n_pages; a.kv_heads = C->kv_heads; a.n_seqs = C->n_seqs; a.n_blocks = C->n_blocks;
    a.page_shift = __builtin_ctz((unsigned)C->page_size);
    a.page_mask = C->page_size - 1;
    return a;
}

// Whether positions' weights [n_seqs, kv_heads, max_len], strides apart, are all places of their own: every sequence's heads together, or every head's sequences.
inline bool weights_apart(const peqa_kv_cache *C, long long max_len, long long seq_stride, long long head_stride)
{
    if (seq_stride < max_len || head_stride < max_len) return false;
    if (C->n_seqs == 1 || C->kv_heads == 1) return true;
    // (n stretches of max_len, `stride` apart, before the next one that is `outer` further: without a product that could overflow)
    auto within = [&](long long n, long long stride, long long outer) { return stride <= (outer - max_len) / (n - 1); };
    return within(C->kv_heads, head_stride, seq_stride) || within(C->n_seqs, seq_stride, head_stride);
}

}  // namespace peqa
