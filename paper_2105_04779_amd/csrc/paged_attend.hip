// Attention of one new token per query row over a sequence's pages of projected keys and values.
//
//   s_t = scale q.K_t (capped, biased by distance),  out = sum_t softmax(s)_t V_t,  lse = log sum_t exp s_t
//
// over the positions that are there: below the length, inside the window, in a page of the pool.
#include <cmath>
#include "paged.h"

namespace el {
namespace {

struct AttendArgs {
    PageView c;
    const int32_t *lengths;
    const char *queries;
    int64_t query_stride;                    // bytes
    const float *slopes;
    float scale, softcap;
    int window, n, beam, heads, kv_heads, d;
    void *out;
    float *lse;
};

// One (query row, head) a workgroup, 256 positions at a time under the running maximum and sum of the softmax.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) k_attend_rows(const AttendArgs a)
{
    __shared__ float q[kMaxHeadDim], p[256], red[8];
    __shared__ int64_t off[256];
    const int tid = threadIdx.x, w = tid >> 6;
    const int head = blockIdx.x % a.heads, m = blockIdx.x / a.heads, b = m / a.beam;
    const int64_t head_off = (int64_t)(head / (a.heads / a.kv_heads)) * a.c.head;
    if (tid < a.d) q[tid] = to_f32(((const T *)(a.queries + m * a.query_stride))[(int64_t)head * a.d + tid]);
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.n) : a.n;
    const float slope = a.slopes ? a.slopes[head] : 0.f;
    float M = -INFINITY, L = 0.f, acc = 0.f;
    for (int t0 = a.window ? max(0, len - a.window) : 0; t0 < len; t0 += 256) {
        __syncthreads();
        const int t = t0 + tid;
        int64_t at = -1;
        float s = -INFINITY;
        if (t < len) {
            const int slot = t / a.c.page_size, page = a.c.table[b * a.c.table_stride + slot];
            if (page >= 0 && page < a.c.pages) {
                at = page * a.c.page + (int64_t)(t - slot * a.c.page_size) * a.c.position + head_off;
                const T *k = (const T *)(a.c.K + at);
                s = 0.f;
                for (int i = 0; i < a.d; ++i) s = fmaf(q[i], to_f32(k[i]), s);
                s *= a.scale;
                if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
                if (a.slopes) s -= slope * (float)(len - 1 - t);
            }
        }
        off[tid] = at;
        float mx = s;
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        if ((tid & 63) == 0) red[w] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(M, fmaxf(red[0], red[1])), fmaxf(red[2], red[3]));
        const float ref = mx == -INFINITY ? 0.f : mx, pr = at < 0 ? 0.f : expf(s - ref);
        float sum = pr;
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        p[tid] = pr;
        if ((tid & 63) == 0) red[4 + w] = sum;
        __syncthreads();
        const float rescale = M == -INFINITY ? 0.f : expf(M - ref);
        L = L * rescale + (red[4] + red[5] + red[6] + red[7]);
        acc *= rescale;
        if (tid < a.d)
            for (int i = 0; i < min(256, len - t0); ++i)
                if (off[i] >= 0) acc = fmaf(p[i], to_f32(((const T *)(a.c.V + off[i]))[tid]), acc);
        M = mx;
    }
    // (no position, or every score -inf: nothing, where the quotient would be 0 / 0; a NaN stays one)
    const bool empty = M == -INFINITY && !(L != L);
    if (tid < a.d) from_f32(empty ? 0.f : acc / L, (TO *)a.out + (int64_t)blockIdx.x * a.d + tid);
    if (tid == 0 && a.lse) a.lse[blockIdx.x] = empty ? -INFINITY : M + logf(L);
}

bool finite_non_negative(float x) { return x >= 0.f && x < INFINITY; }

} // namespace
} // namespace el

extern "C" size_t el_attn_paged_workspace_bytes(const el_attn_pages *cache, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    if (el::check_pages(cache) != EL_OK || heads < 1 || B < 1 || beam < 1 || n < 1) return 0;
    return 0;
}

extern "C" el_status el_attn_paged_attend(const el_attn_pages *cache,
                                          const int32_t *table, int64_t table_stride, int32_t table_pages, const int32_t *lengths,
                                          const void *queries, int64_t query_stride, int32_t heads, const el_attn_score_rule *rule,
                                          void *out, int32_t out_dtype, float *lse, int32_t B, int32_t beam, int32_t n,
                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (const el_status st = check_pages(cache); st != EL_OK) return st;
    if (const el_status st = check_table(table, table_stride, table_pages, B); st != EL_OK) return st;
    if (!queries || !rule || !out || heads < 1 || beam < 1 || n < 1) return EL_ERR_INVALID_ARG;
    if (out_dtype != EL_F32 && out_dtype != cache->dtype) return EL_ERR_UNSUPPORTED;
    if (heads % cache->kv_heads != 0 || n > (int64_t)table_pages * cache->page_size) return EL_ERR_INVALID_ARG;
    if (!(fabsf(rule->scale) < INFINITY) || !finite_non_negative(rule->softcap) || rule->window < 0) return EL_ERR_INVALID_ARG;
    const int64_t es = (int64_t)dtype_size(cache->dtype), row = (int64_t)heads * cache->d_head, rows = (int64_t)B * beam;
    if (((uintptr_t)lengths | (uintptr_t)lse | (uintptr_t)rule->slopes) & 3 || ((uintptr_t)queries | (uintptr_t)out) & 15) return EL_ERR_INVALID_ARG;
    if (query_stride > ((int64_t)1 << 44) || query_stride * es % 16 != 0 || (rows > 1 && query_stride < row)) return EL_ERR_INVALID_ARG;
    if (rows * heads > INT32_MAX) return EL_ERR_INVALID_ARG;
    const AttendArgs a{page_view(*cache, table, table_stride, table_pages), lengths, (const char *)queries, query_stride * es, rule->slopes,
                       rule->scale, rule->softcap, rule->window, n, beam, heads, cache->kv_heads, cache->d_head, out, lse};
    const dim3 grid((unsigned)(rows * heads)), block(256);
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    if (cache->dtype == EL_F32) hipLaunchKernelGGL((k_attend_rows<float, float>), grid, block, 0, s, a);
    else if (cache->dtype == EL_F16 && out_dtype == EL_F16) hipLaunchKernelGGL((k_attend_rows<f16_t, f16_t>), grid, block, 0, s, a);
    else if (cache->dtype == EL_F16) hipLaunchKernelGGL((k_attend_rows<f16_t, float>), grid, block, 0, s, a);
    else if (out_dtype == EL_BF16) hipLaunchKernelGGL((k_attend_rows<bf16_t, bf16_t>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_attend_rows<bf16_t, float>), grid, block, 0, s, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}
