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
    int per_row, rows_on, pieces_on;             // pieces of 16 bytes of a token's head; whole rows, and pieces beyond them, that 64 pieces are
};

typedef short s2v __attribute__((ext_vector_type(2)));

// 16 bytes of new values.  Size: the largest |value| by its bits, which order like it.  With kGap added infinities and NaN alone are negative: they never are
// the largest, and the sign of `all` tells of them.
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
    static constexpr int N = 4;
    static constexpr unsigned kGap = 0x00800000u;
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(v[i]); }
    struct Size {
        int top = (int)kGap, all = 0;
        __device__ __forceinline__ void add(u4 v)
        {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = (int)((v[i] & 0x7fffffffu) + kGap);
                top = max(top, x);
                all |= x;
            }
        }
        __device__ __forceinline__ float most() const { return __uint_as_float((unsigned)top - kGap); }
        __device__ __forceinline__ bool special() const { return all < 0; }
    };
};
template <typename T, unsigned GAP> struct Sixteen16 {
    static constexpr int N = 8;
    struct Size {
        s2v top = {(short)GAP, (short)GAP};
        unsigned all = 0;
        __device__ __forceinline__ void add(u4 v)
        {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned w = v[i] & 0x7fff7fffu;
                const s2v x = __builtin_bit_cast(s2v, w) + s2v{(short)GAP, (short)GAP};
                top = __builtin_elementwise_max(top, x);
                all |= __builtin_bit_cast(unsigned, x);
            }
        }
        __device__ __forceinline__ float most() const
        {
            const unsigned bits = (unsigned)(max((int)top[0], (int)top[1]) - (int)GAP);
            const u4 v = {bits, 0, 0, 0};
            return Sixteen<T>::at(v, 0);
        }
        __device__ __forceinline__ bool special() const { return (all & 0x80008000u) != 0; }
    };
};
template <> struct Sixteen<bf16_t> : Sixteen16<bf16_t, 0x0080> {
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
};
template <> struct Sixteen<f16_t> : Sixteen16<f16_t, 0x0400> {
    static __device__ __forceinline__ float at(u4 v, int i) { const unsigned u = v[i >> 1]; return (float)__builtin_bit_cast(h2, u)[i & 1]; }
};

// One wavefront a (sequence, block that receives tokens, head, K or V): the largest of its new tokens, then their codes.  Grid: (blocks x heads x 2 / 4, B).
// Bound by HBM: new values are read once where HOLD pieces a lane hold them.  The vector ALU would take longer than the memory with a conversion and a comparison for
// each value's size, clamps for infinities that are hardly ever there and a division for each piece's place, so sizes are found two at once from the bits,
// blocks without infinities and NaN take no clamps (a value times the reciprocal is at most `most` (1 + 2^-22), which rounds to it), and places follow one
// another by addition: 16 prompts of 2048 in fp16, 8 heads of 128, blocks of 32, 35 us (5.7 TB/s); three passes a captured graph 40 (45 with new values kept in the
// caches), 100 without all that.
template <int FMT, typename T>
__global__ void __launch_bounds__(256, 5) k_append8(const Append8Args a)
{
    typedef Sixteen<T> P;
    constexpr int N = P::N, HOLD = 8;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y, is_v = (int)(unit & 1), h = (int)((unsigned)(unit >> 1) % (unsigned)a.kv_heads), nth = (int)((unsigned)(unit >> 1) / (unsigned)a.kv_heads);
    if (nth >= a.blocks) return;
    const int count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    const int64_t len = a.lengths[b], start = len - count, begin = start > 0 ? start : 0;
    const int block = a.s.block;
    const int64_t base = ((int64_t)((unsigned)begin / (unsigned)block) + nth) * block, lo = base > begin ? base : begin, hi = base + block < len ? base + block : len;
    if (lo >= hi || base >= (int64_t)a.c.table_pages * a.c.page_size) return;
    const int slot = (int)((unsigned)base / (unsigned)a.c.page_size), off = (int)(base - (int64_t)slot * a.c.page_size);
    const int page = a.c.table[b * a.c.table_stride + slot];
    if (page < 0 || page >= a.c.pages) return;

    const int total = (int)(hi - lo) * a.per_row;                    // pieces of 16 bytes
    const char *const from = (is_v ? a.V_new : a.K_new) + b * a.batch_stride + (lo - start) * a.token_stride + (int64_t)h * a.d * (int)sizeof(T);
    char *const codes = (is_v ? a.c.V : a.c.K) + page * a.c.page + off * a.c.position + h * a.c.head;       // of the block's first position
    float *const scale_at = (is_v ? a.s.V : a.s.K) + ((int64_t)page * a.kv_heads + h) * a.s.per + a.s.by_block.of(off);
    const int had = start > base ? (int)(start - base) : 0;          // earlier positions of the block
    const float old = had ? *scale_at : 0.f;
    // pieces lane, lane + 64, ..: where they are in rows a stride apart
    const int row0 = (int)((unsigned)lane / (unsigned)a.per_row), col0 = lane - row0 * a.per_row;
    struct Way { int k, col; int64_t at; };
    auto first = [&](int64_t stride, int width) __attribute__((always_inline)) { return Way{lane, col0, row0 * stride + col0 * width}; };
    auto next = [&](Way &w, int64_t stride, int width) __attribute__((always_inline)) {
        w.k += 64;
        w.col += a.pieces_on;
        w.at += a.rows_on * stride + a.pieces_on * width;
        const bool over = w.col >= a.per_row;
        w.col -= over ? a.per_row : 0;
        w.at += over ? stride - a.per_row * width : 0;
    };
    u4 held[HOLD];
    typename P::Size size;
    Way r = first(a.token_stride, 16);
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
        held[j] = u4{0, 0, 0, 0};
        if (r.k < total) held[j] = __builtin_nontemporal_load((const u4 *)(from + r.at));
        next(r, a.token_stride, 16);
    }
#pragma unroll
    for (int j = 0; j < HOLD; ++j) size.add(held[j]);
#pragma unroll 1
    for (; r.k < total; next(r, a.token_stride, 16)) size.add(*(const u4 *)(from + r.at));
    float most = size.most();
    const bool special = __ballot(size.special()) != 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
    const float needed = fmaxf(most * (1.f / Code<FMT>::most), kSmallestScale);
    const bool grows = needed > old, keeps = had && !grows;
    const float scale = keeps ? old : needed, inverse = 1.f / scale;
    if (had && grows) {
        const int chunks = a.d / 16;
#pragma unroll 1
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
    char *const to = codes + (lo - base) * a.c.position;
    Way w = first(a.c.position, N);
    auto store = [&](u4 v, auto clamped) __attribute__((always_inline)) {
        unsigned x[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float y0 = P::at(v, 4 * i) * inverse, y1 = P::at(v, 4 * i + 1) * inverse, y2 = P::at(v, 4 * i + 2) * inverse, y3 = P::at(v, 4 * i + 3) * inverse;
            if constexpr (decltype(clamped)::value) x[i] = Code<FMT>::of4(y0, y1, y2, y3);
            else x[i] = Code<FMT>::of4_inside(y0, y1, y2, y3);
        }
        if constexpr (N == 8) *(u2 *)(to + w.at) = u2{x[0], x[1]};
        else *(unsigned *)(to + w.at) = x[0];
    };
    if (!special) {
#pragma unroll
        for (int j = 0; j < HOLD; ++j) {
            if (w.k < total) store(held[j], std::false_type{});
            next(w, a.c.position, N);
        }
    } else {
        w.k = lane;
    }
    // pieces that were not held, or all of a block with infinities or NaN, once more from memory
    r = first(a.token_stride, 16);
    if (!special)
#pragma unroll
        for (int j = 0; j < HOLD; ++j) next(r, a.token_stride, 16);
#pragma unroll 1
    for (; w.k < total; next(w, a.c.position, N), next(r, a.token_stride, 16)) store(*(const u4 *)(from + r.at), std::true_type{});
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
    if (groups >= 1 << 24 || groups * B > INT32_MAX) return EL_ERR_UNSUPPORTED;                      // (a launch has fewer than 2^32 lanes a dimension)
    const int per_row = cache->d_head * (int)es / 16;
    const Append8Args a{page_view8(*cache, table, table_stride, table_pages), scale_view(*cache), lengths, counts, (const char *)K_new, (const char *)V_new,
                        batch_stride * es, token_stride * es, cache->kv_heads, cache->d_head, T, (int)blocks, per_row, 64 / per_row, 64 % per_row};
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
