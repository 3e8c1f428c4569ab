// The paged key/value cache between attentions: new tokens into their pages, and copies of pages for beams that fork.
// Pure data movement in pieces of 16 bytes: every byte is read once and written once.
#include "paged.h"

namespace el {

el_status check_layout(const void *K, const void *V, int64_t page_stride, int64_t position_stride, int64_t head_stride,
                       int32_t pages, int32_t page_size, int32_t kv_heads, int32_t d_head, int64_t es)
{
    if (pages < 1 || page_size < 1 || kv_heads < 1 || d_head < 1) return EL_ERR_INVALID_ARG;
    if (d_head > kMaxHeadDim || d_head * es % 16 != 0) return EL_ERR_UNSUPPORTED;
    // strides: multiples of 16 bytes, and no two elements in one place: each axis steps over all that the smaller steps cover
    struct Axis { int64_t size, stride; } ax[3] = {{pages, page_stride}, {page_size, position_stride}, {kv_heads, head_stride}};
    for (const Axis &a : ax)
        if (a.stride < 0 || a.stride > ((int64_t)1 << 44) || a.stride * es % 16 != 0) return EL_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (ax[j].stride > ax[j + 1].stride) { const Axis t = ax[j]; ax[j] = ax[j + 1]; ax[j + 1] = t; }
    __int128 extent = d_head;
    for (const Axis &a : ax) {
        if (a.size == 1) continue;
        if (a.stride < extent) return EL_ERR_INVALID_ARG;
        extent = (__int128)a.stride * (a.size - 1) + extent;
    }
    if (extent * es > ((__int128)1 << 48)) return EL_ERR_INVALID_ARG;
    if (((uintptr_t)K | (uintptr_t)V) & 15) return EL_ERR_INVALID_ARG;
    return EL_OK;
}

el_status check_pages(const el_attn_pages *c)
{
    if (!c || !c->K || !c->V) return EL_ERR_INVALID_ARG;
    if (c->dtype != EL_F32 && c->dtype != EL_F16 && c->dtype != EL_BF16) return EL_ERR_UNSUPPORTED;
    return check_layout(c->K, c->V, c->page_stride, c->position_stride, c->head_stride, c->pages, c->page_size, c->kv_heads, c->d_head,
                        (int64_t)dtype_size(c->dtype));
}

el_status check_table(const int32_t *table, int64_t table_stride, int32_t table_pages, int32_t B)
{
    if (!table || table_pages < 1 || B < 1 || table_stride < table_pages || table_stride > ((int64_t)1 << 40)) return EL_ERR_INVALID_ARG;
    if ((uintptr_t)table & 3 || out_of_reach(B, table_stride * 4)) return EL_ERR_INVALID_ARG;
    return EL_OK;
}

el_status check_new_tokens(const int32_t *lengths, const int32_t *counts, const void *K_new, const void *V_new, int64_t batch_stride, int64_t token_stride,
                           int64_t row, int64_t es, int32_t B, int32_t T)
{
    if (!lengths || !K_new || !V_new || T < 1 || T > 1 << 23 || B > 65535) return EL_ERR_INVALID_ARG;        // (grid)
    if (((uintptr_t)lengths | (uintptr_t)counts) & 3 || ((uintptr_t)K_new | (uintptr_t)V_new) & 15) return EL_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 44;
    if (token_stride > most || batch_stride > most || token_stride * es % 16 != 0 || batch_stride * es % 16 != 0) return EL_ERR_INVALID_ARG;
    if ((T > 1 && token_stride < row) || (B > 1 && batch_stride < row)) return EL_ERR_INVALID_ARG;
    if (row * es / 16 > INT32_MAX - 256 || out_of_reach(T, token_stride * es) || out_of_reach(B, batch_stride * es)) return EL_ERR_INVALID_ARG;
    return EL_OK;
}

el_status check_pairs(const int32_t *src, const int32_t *dst, const int32_t *counts, int32_t pairs)
{
    if (!src || !dst || pairs < 1 || pairs > 1 << 23) return EL_ERR_INVALID_ARG;
    return ((uintptr_t)src | (uintptr_t)dst | (uintptr_t)counts) & 3 ? EL_ERR_INVALID_ARG : EL_OK;
}

PageView page_view(const el_attn_pages &c, const int32_t *table, int64_t table_stride, int table_pages)
{
    const int64_t es = (int64_t)dtype_size(c.dtype);
    return PageView{(char *)c.K, (char *)c.V, c.page_stride * es, c.position_stride * es, c.head_stride * es,
                    table, table_stride, table_pages, c.pages, c.page_size};
}

namespace {

typedef unsigned int u4v __attribute__((ext_vector_type(4)));

struct AppendArgs {
    PageView c;
    const int32_t *lengths, *counts;
    const char *K_new, *V_new;
    int64_t batch_stride, token_stride;      // bytes
    int kv_heads, chunks, T;                 // chunks: pieces of 16 bytes of a head
    int lanes;                               // of a token that shares its workgroup: a power of 2
};

// Grid: (T, B), a token a workgroup; SHARED: small tokens, 256 / lanes of them a workgroup: 64 x 512 of one head of 64 in bf16 4.1 us, 20.5 alone; of
// two of 128 16.3 / 25.9; 8192 of eight of 128, two a workgroup, 15.9 / 15.2.
template <bool SHARED>
__global__ void __launch_bounds__(256) k_append(const AppendArgs a)
{
    const int lanes = SHARED ? a.lanes : 256, lane = threadIdx.x & (lanes - 1), b = blockIdx.y;
    const int i = SHARED ? blockIdx.x * (256 / lanes) + threadIdx.x / lanes : blockIdx.x;
    const int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    const int64_t at = (int64_t)a.lengths[b] - count + i;
    if (i >= count || at < 0 || at >= (int64_t)a.c.table_pages * a.c.page_size) return;
    const int slot = (int)(at / a.c.page_size);
    const int page = a.c.table[b * a.c.table_stride + slot];
    if (page < 0 || page >= a.c.pages) return;
    const int64_t from = b * a.batch_stride + i * a.token_stride;
    const int64_t to = page * a.c.page + (at - (int64_t)slot * a.c.page_size) * a.c.position;
    const int total = a.kv_heads * a.chunks;
    for (int k = lane; k < total; k += lanes) {
        const int64_t d = to + (k / a.chunks) * a.c.head + (k % a.chunks) * 16;
        *(u4v *)(a.c.K + d) = *(const u4v *)(a.K_new + from + (int64_t)k * 16);
        *(u4v *)(a.c.V + d) = *(const u4v *)(a.V_new + from + (int64_t)k * 16);
    }
}

struct CopyArgs {
    PageView c;
    const int32_t *src, *dst, *counts;
    unsigned kv_heads, chunks;
    int heads_first;                         // a head's positions lie closer together than a position's heads
    float *K_scale, *V_scale;                // SCALES: [pages, kv_heads, per], `block` positions each
    unsigned block, per;
};

// Grid: (pairs, slices of a page).  Bound by HBM: four pieces of K and of V on their way per lane, stored past the caches: 2048 pages of 64
// positions, 16 heads of 64 in bf16, half full on average, 114 us for 545 MB = 4.8 TB/s of reads and writes; 512 of 16 positions 7.6 us (8.8 with
// stores that stay in the caches).
template <bool SCALES>
__global__ void __launch_bounds__(256) k_copy(const CopyArgs a)
{
    const int src = a.src[blockIdx.x], dst = a.dst[blockIdx.x];
    if (src < 0 || src >= a.c.pages || dst < 0 || dst >= a.c.pages || src == dst) return;
    const unsigned count = a.counts ? min(max(a.counts[blockIdx.x], 0), a.c.page_size) : a.c.page_size;
    const unsigned total = count * a.kv_heads * a.chunks, inner = (a.heads_first ? count : a.kv_heads) * a.chunks;
    const int64_t outer_step = a.heads_first ? a.c.head : a.c.position, inner_step = a.heads_first ? a.c.position : a.c.head;
    const char *const Ks = a.c.K + src * a.c.page, *const Vs = a.c.V + src * a.c.page;
    char *const Kd = a.c.K + dst * a.c.page, *const Vd = a.c.V + dst * a.c.page;
    // pieces in the order of memory, as far as the strides allow
    auto place = [&](unsigned k) {
        const unsigned o = k / inner, r = k - o * inner, i = r / a.chunks;
        return o * outer_step + i * inner_step + (r - i * a.chunks) * 16;
    };
    constexpr int AHEAD = 4;
    for (unsigned k0 = blockIdx.y * (256 * AHEAD); k0 < total; k0 += gridDim.y * (256 * AHEAD)) {
        u4v kk[AHEAD], vv[AHEAD];
        int64_t at[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const unsigned k = k0 + j * 256 + threadIdx.x;
            at[j] = k < total ? place(k) : -1;
            if (at[j] >= 0) { kk[j] = *(const u4v *)(Ks + at[j]); vv[j] = *(const u4v *)(Vs + at[j]); }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (at[j] >= 0) { __builtin_nontemporal_store(kk[j], (u4v *)(Kd + at[j])); __builtin_nontemporal_store(vv[j], (u4v *)(Vd + at[j])); }
    }
    if constexpr (SCALES) {
        // those of the blocks that the positions begin or fill, by the pair's last slice, which has the fewest pieces
        if (blockIdx.y != gridDim.y - 1) return;
        const unsigned used = (count + a.block - 1) / a.block;
        const int64_t page = (int64_t)a.kv_heads * a.per;
        for (unsigned k = threadIdx.x; k < used * a.kv_heads; k += 256) {
            const unsigned h = k / used, at = h * a.per + (k - h * used);
            a.K_scale[dst * page + at] = a.K_scale[src * page + at];
            a.V_scale[dst * page + at] = a.V_scale[src * page + at];
        }
    }
}

} // namespace

el_status launch_copy(const PageView &c, const int32_t *src, const int32_t *dst, const int32_t *counts, int32_t pairs, int kv_heads, int head_bytes,
                      float *K_scale, float *V_scale, int block, void *stream)
{
    const int64_t chunks = head_bytes / 16, pieces = (int64_t)c.page_size * kv_heads * chunks;
    if (pieces > INT32_MAX) return EL_ERR_UNSUPPORTED;
    const CopyArgs a{c, src, dst, counts, (unsigned)kv_heads, (unsigned)chunks, c.position < c.head, K_scale, V_scale, (unsigned)block,
                     (unsigned)(block ? c.page_size / block : 0)};
    // slices of 1024 pieces, most of them a workgroup's only one (2048 of those pages: 125 us with 2048 workgroups, 114 with 16384)
    const int64_t most = (pieces + 1023) / 1024, want = (32768 + pairs - 1) / pairs;
    const dim3 grid(pairs, (unsigned)(most < want ? most : want));
    (void)hipGetLastError();
    if (block) hipLaunchKernelGGL(k_copy<true>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(k_copy<false>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}

} // namespace el

extern "C" el_status el_attn_paged_append(const el_attn_pages *cache,
                                          const int32_t *table, int64_t table_stride, int32_t table_pages,
                                          const int32_t *lengths, const int32_t *counts,
                                          const void *K_new, const void *V_new, int64_t batch_stride, int64_t token_stride,
                                          int32_t B, int32_t T, void *stream)
{
    if (const el_status st = el::check_pages(cache); st != EL_OK) return st;
    if (const el_status st = el::check_table(table, table_stride, table_pages, B); st != EL_OK) return st;
    const int64_t es = (int64_t)el::dtype_size(cache->dtype), row = (int64_t)cache->kv_heads * cache->d_head;
    if (const el_status st = el::check_new_tokens(lengths, counts, K_new, V_new, batch_stride, token_stride, row, es, B, T); st != EL_OK) return st;
    int lanes = 1;
    while (lanes < 128 && lanes < row * es / 16) lanes *= 2;
    const el::AppendArgs a{el::page_view(*cache, table, table_stride, table_pages), lengths, counts, (const char *)K_new, (const char *)V_new,
                           batch_stride * es, token_stride * es, cache->kv_heads, (int)(cache->d_head * es / 16), T, lanes};
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    const int tokens = 256 / lanes;
    if (tokens > 2) hipLaunchKernelGGL(el::k_append<true>, dim3((T + tokens - 1) / tokens, B), dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(el::k_append<false>, dim3(T, B), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}

extern "C" el_status el_attn_paged_copy(const el_attn_pages *cache, const int32_t *src, const int32_t *dst, const int32_t *counts,
                                        int32_t pairs, void *stream)
{
    if (const el_status st = el::check_pages(cache); st != EL_OK) return st;
    if (const el_status st = el::check_pairs(src, dst, counts, pairs); st != EL_OK) return st;
    return el::launch_copy(el::page_view(*cache, nullptr, 0, 0), src, dst, counts, pairs, cache->kv_heads, (int)(cache->d_head * el::dtype_size(cache->dtype)),
                           nullptr, nullptr, 0, stream);
}
