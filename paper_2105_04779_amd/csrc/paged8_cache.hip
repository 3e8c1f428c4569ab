// The paged cache in 8 bits between attentions: new tokens rounded to codes with a scale for each block of positions and head, and copies of pages.
#include "paged8.h"

namespace el {

el_status check_pages8(const el_attn_pages8 *c)
{
    if (!c || !c->K || !c->V || !c->K_scale || !c->V_scale) return EL_ERR_INVALID_ARG;
    if (c->format != EL_E4M3 && c->format != EL_INT8) return EL_ERR_UNSUPPORTED;
    if (const el_status st = check_layout(c->K, c->V, c->page_stride, c->position_stride, c->head_stride, c->pages, c->page_size, c->kv_heads, c->d_head, 1);
        st != EL_OK) return st;
    if (c->page_size > kMaxPage8) return EL_ERR_UNSUPPORTED;
    if (c->block < 1 || c->page_size % c->block != 0 || ((uintptr_t)c->K_scale | (uintptr_t)c->V_scale) & 3) return EL_ERR_INVALID_ARG;
    const __int128 scales = (__int128)c->pages * c->kv_heads * (c->page_size / c->block);
    return scales > ((__int128)1 << 46) ? EL_ERR_INVALID_ARG : EL_OK;
}

PageView page_view8(const el_attn_pages8 &c, const int32_t *table, int64_t table_stride, int table_pages)
{
    return PageView{(char *)c.K, (char *)c.V, c.page_stride, c.position_stride, c.head_stride, table, table_stride, table_pages, c.pages, c.page_size};
}

namespace {

constexpr float kSmallestScale = 0x1p-126f;      // its reciprocal is a number

struct Append8Args {
    PageView c;
    ScaleView s;
    const int32_t *lengths, *counts;
    const char *K_new, *V_new;
    int64_t batch_stride, token_stride;          // bytes
    int kv_heads, d, T, blocks;                  // blocks: that T tokens may touch
};

template <typename T> struct Sixteen;            // 16 bytes of new values
template <> struct Sixteen<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(v[i]); }
};
template <> struct Sixteen<bf16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
};
template <> struct Sixteen<f16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float at(u4 v, int i) { const unsigned u = v[i >> 1]; return (float)__builtin_bit_cast(h2, u)[i & 1]; }
};

// One wavefront a (sequence, block that receives tokens, head, K or V): the largest of its new tokens, then their codes.  Grid: (blocks x heads x 2 / 4, B).
// Bound by HBM: new values are read once where HOLD pieces a lane hold them.
template <int FMT, typename T>
__global__ void __launch_bounds__(256) k_append8(const Append8Args a)
{
    typedef Sixteen<T> P;
    constexpr int N = P::N, HOLD = 8;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int b = blockIdx.y, is_v = (int)(unit & 1), h = (int)((unit >> 1) % a.kv_heads);
    const int64_t nth = (unit >> 1) / a.kv_heads;
    if (nth >= a.blocks) return;
    const int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    const int64_t len = a.lengths[b], start = len - count, begin = start > 0 ? start : 0;
    const int block = a.s.block;
    const int64_t base = (begin / block + nth) * block, lo = base > begin ? base : begin, hi = base + block < len ? base + block : len;
    if (lo >= hi || base >= (int64_t)a.c.table_pages * a.c.page_size) return;
    const int slot = (int)(base / a.c.page_size), off = (int)(base - (int64_t)slot * a.c.page_size);
    const int page = a.c.table[b * a.c.table_stride + slot];
    if (page < 0 || page >= a.c.pages) return;

    const int per_row = a.d / N, total = (int)(hi - lo) * per_row;   // pieces of 16 bytes
    const char *const from = (is_v ? a.V_new : a.K_new) + b * a.batch_stride + (lo - start) * a.token_stride + (int64_t)h * a.d * (int)sizeof(T);
    char *const codes = (is_v ? a.c.V : a.c.K) + page * a.c.page + off * a.c.position + h * a.c.head;       // of the block's first position
    float *const scale_at = (is_v ? a.s.V : a.s.K) + ((int64_t)page * a.kv_heads + h) * a.s.per + a.s.by_block.of(off);
    auto load = [&](int k) __attribute__((always_inline)) { const int row = k / per_row; return *(const u4 *)(from + row * a.token_stride + (k - row * per_row) * 16); };
    float most = 0.f;
    auto larger = [&](u4 v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) { const float x = fabsf(P::at(v, i)); most = fmaxf(most, x < INFINITY ? x : 0.f); }
    };
    u4 held[HOLD];
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
        held[j] = u4{0, 0, 0, 0};
        if (lane + 64 * j < total) held[j] = load(lane + 64 * j);
    }
#pragma unroll
    for (int j = 0; j < HOLD; ++j) larger(held[j]);
    for (int k = lane + 64 * HOLD; k < total; k += 64) larger(load(k));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
    const float needed = fmaxf(most * (1.f / Code<FMT>::most), kSmallestScale);
    const int had = start > base ? (int)(start - base) : 0;          // earlier positions of the block
    const float old = had ? *scale_at : 0.f;
    const bool grows = needed > old, keeps = had && !grows;
    const float scale = keeps ? old : needed, inverse = 1.f / scale;
    if (had && grows) {
        const int chunks = a.d / 16;
        for (int k = lane; k < had * chunks; k += 64) {
            const int row = k / chunks;
            u4 *const at = (u4 *)(codes + row * a.c.position + (k - row * chunks) * 16);
            u4 v = *at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f4 x = Code<FMT>::values(v[i]);
                v[i] = Code<FMT>::of4(x[0] * old * inverse, x[1] * old * inverse, x[2] * old * inverse, x[3] * old * inverse);
            }
            *at = v;
        }
    }
    auto store = [&](int k, u4 v) __attribute__((always_inline)) {
        const int row = k / per_row;
        char *const at = codes + (lo - base + row) * a.c.position + (k - row * per_row) * N;
        unsigned w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            w[i] = Code<FMT>::of4(P::at(v, 4 * i) * inverse, P::at(v, 4 * i + 1) * inverse, P::at(v, 4 * i + 2) * inverse, P::at(v, 4 * i + 3) * inverse);
        if constexpr (N == 8) *(u2 *)at = u2{w[0], w[1]};
        else *(unsigned *)at = w[0];
    };
#pragma unroll
    for (int j = 0; j < HOLD; ++j)
        if (lane + 64 * j < total) store(lane + 64 * j, held[j]);
    for (int k = lane + 64 * HOLD; k < total; k += 64) store(k, load(k));
    if (lane == 0 && !keeps) *scale_at = scale;
}

template <int FMT>
void launch_append8(const Append8Args &a, int dtype, dim3 grid, hipStream_t s)
{
    if (dtype == EL_F32) hipLaunchKernelGGL((k_append8<FMT, float>), grid, dim3(256), 0, s, a);
    else if (dtype == EL_F16) hipLaunchKernelGGL((k_append8<FMT, f16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_append8<FMT, bf16_t>), grid, dim3(256), 0, s, a);
}

} // namespace
} // namespace el

extern "C" el_status el_attn_quantized_append(const el_attn_pages8 *cache, int32_t dtype,
                                              const int32_t *table, int64_t table_stride, int32_t table_pages,
                                              const int32_t *lengths, const int32_t *counts,
                                              const void *K_new, const void *V_new, int64_t batch_stride, int64_t token_stride,
                                              int32_t B, int32_t T, void *stream)
{
    using namespace el;
    if (const el_status st = check_pages8(cache); st != EL_OK) return st;
    if (dtype != EL_F32 && dtype != EL_F16 && dtype != EL_BF16) return EL_ERR_UNSUPPORTED;
    if (const el_status st = check_table(table, table_stride, table_pages, B); st != EL_OK) return st;
    if (const el_status st = check_new_tokens(lengths, counts, K_new, V_new, batch_stride, token_stride, (int64_t)cache->kv_heads * cache->d_head,
                                              (int64_t)dtype_size(dtype), B, T); st != EL_OK) return st;
    const int64_t es = (int64_t)dtype_size(dtype), blocks = ((int64_t)T + cache->block - 2) / cache->block + 1;
    const int64_t groups = (blocks * cache->kv_heads * 2 + 3) / 4;
    if (groups > INT32_MAX || groups * B > INT32_MAX) return EL_ERR_UNSUPPORTED;                     // (grid)
    const Append8Args a{page_view8(*cache, table, table_stride, table_pages), scale_view(*cache), lengths, counts, (const char *)K_new, (const char *)V_new,
                        batch_stride * es, token_stride * es, cache->kv_heads, cache->d_head, T, (int)blocks};
    const dim3 grid((unsigned)groups, (unsigned)B);
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    if (cache->format == EL_E4M3) launch_append8<EL_E4M3>(a, dtype, grid, (hipStream_t)stream);
    else launch_append8<EL_INT8>(a, dtype, grid, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}

extern "C" el_status el_attn_quantized_copy(const el_attn_pages8 *cache, const int32_t *src, const int32_t *dst, const int32_t *counts,
                                            int32_t pairs, void *stream)
{
    if (const el_status st = el::check_pages8(cache); st != EL_OK) return st;
    if (const el_status st = el::check_pairs(src, dst, counts, pairs); st != EL_OK) return st;
    return el::launch_copy(el::page_view8(*cache, nullptr, 0, 0), src, dst, counts, pairs, cache->kv_heads, cache->d_head, cache->K_scale, cache->V_scale,
                           cache->block, stream);
}
