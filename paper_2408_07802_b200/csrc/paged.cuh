// What the kernels on the paged key/value cache share: the cache's description and the checked page lookup.
#pragma once
#include "internal.h"
#include "ptx.cuh"

namespace kr {

struct PagedView {
    uint16_t *k, *v;
    const int *table;
    long long page_stride, head_stride, slot_stride, table_stride;
    int n_pages, page_size, n_kv_head, n_seqs, max_pages;
};

// Argument checks that do not touch the device; fills the view.
inline int paged_view(const kraken_paged_cache *c, PagedView *v) {
    if (!c || !c->k || !c->v || !c->page_table || c->n_pages < 1 || c->page_size < 1 || c->n_kv_head < 1 ||
        c->n_seqs < 1 || c->max_pages < 1 || c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0 ||
        c->table_stride < c->max_pages || (long long)c->max_pages * c->page_size > 0x7fffff00LL)
        return KRAKEN_EINVAL;
    if (!decode_head_dim_ok(c->head_dim)) return KRAKEN_EUNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(c->k) & 15) || (reinterpret_cast<uintptr_t>(c->v) & 15) || (c->page_stride & 7) ||
        (c->head_stride & 7) || (c->slot_stride & 7))
        return KRAKEN_EUNSUPPORTED;
    v->k = static_cast<uint16_t *>(c->k);
    v->v = static_cast<uint16_t *>(c->v);
    v->table = c->page_table;
    v->page_stride = c->page_stride;
    v->head_stride = c->head_stride;
    v->slot_stride = c->slot_stride;
    v->table_stride = c->table_stride;
    v->n_pages = c->n_pages;
    v->page_size = c->page_size;
    v->n_kv_head = c->n_kv_head;
    v->n_seqs = c->n_seqs;
    v->max_pages = c->max_pages;
    return KRAKEN_OK;
}

constexpr uint32_t STATUS_BAD_PAGE = KRAKEN_STATUS_BAD_PAGE;

}  // namespace kr
