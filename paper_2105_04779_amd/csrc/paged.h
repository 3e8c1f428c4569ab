// What the calls on a paged key/value cache share: the checks of their arguments and the way from a position to its storage.
#pragma once
#include "el_internal.h"

namespace el {

constexpr int kMaxHeadDim = 256;

// Host: EL_OK if the cache is one that the kernels cover (el_attn.h states the rules).
el_status check_pages(const el_attn_pages *c);
// Host: table, rows and lengths as every call takes them.
el_status check_table(const int32_t *table, int64_t table_stride, int32_t table_pages, int32_t B);

// The cache as kernels see it: strides in bytes.
struct PageView {
    char *K, *V;
    int64_t page, position, head;
    const int32_t *table;
    int64_t table_stride;
    int table_pages, pages, page_size;
};
PageView page_view(const el_attn_pages &c, const int32_t *table, int64_t table_stride, int table_pages);

} // namespace el
