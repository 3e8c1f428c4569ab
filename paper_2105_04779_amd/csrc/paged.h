// What the calls on a paged key/value cache share: the checks of their arguments and the way from a position to its storage.
#pragma once
#include "el_internal.h"

namespace el {

constexpr int kMaxHeadDim = 256;

// Host: EL_OK if the cache is one that the kernels cover (el_attn.h states the rules).
el_status check_pages(const el_attn_pages *c);
// Host: where pools of elements of `es` bytes lie: sizes, strides, alignment.
el_status check_layout(const void *K, const void *V, int64_t page_stride, int64_t position_stride, int64_t head_stride,
                       int32_t pages, int32_t page_size, int32_t kv_heads, int32_t d_head, int64_t es);
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
// Host: the operands of append and of copy, for rows of `row` elements of `es` bytes.
el_status check_new_tokens(const int32_t *lengths, const int32_t *counts, const void *K_new, const void *V_new, int64_t batch_stride, int64_t token_stride,
                           int64_t row, int64_t es, int32_t B, int32_t T);
el_status check_pairs(const int32_t *src, const int32_t *dst, const int32_t *counts, int32_t pairs);
// Host: launches the copies of pages; arguments have been checked.  With `block`, the scales [pages, kv_heads, page_size / block] of the blocks too.
el_status launch_copy(const PageView &c, const int32_t *src, const int32_t *dst, const int32_t *counts, int32_t pairs, int kv_heads, int head_bytes,
                      float *K_scale, float *V_scale, int block, void *stream);
PageView page_view(const el_attn_pages &c, const int32_t *table, int64_t table_stride, int table_pages);

} // namespace el
