// What a row of logits says about the next token: log-probability of a given one, entropy, the best alternatives.
//
//   lse = m + log S,  S = sum exp(x - m),  entropy = log S - T / S,  T = sum exp(x - m) (x - m),  m the largest logit
#include <cmath>
#include "el_internal.h"

namespace el {
namespace {

constexpr int kMaxAlternatives = 64;

struct ScoreArgs {
    const char *logits;
    int64_t row_stride;          // elements
    int vocab, k;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_index;
};

// What orders alternatives: the value, then the lower index.  0: no alternative (-inf or NaN).
__device__ __forceinline__ unsigned long long order_key(float x, int v)
{
    if (!(x > -INFINITY)) return 0ull;
    const unsigned u = __float_as_uint(x + 0.f);                     // (-0 counts as 0)
    return ((unsigned long long)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32) | (0xffffffffu - (unsigned)v);
}
__device__ __forceinline__ float key_value(unsigned long long key)
{
    const unsigned u = (unsigned)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V *red, F f)
{
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return f(f(red[0], red[1]), f(red[2], red[3]));
}

// One row a workgroup; one pass for the maximum, one for the sums, one for every alternative.
template <typename T>
__global__ void __launch_bounds__(256) k_score_rows(const ScoreArgs a)
{
    __shared__ float red[4];
    __shared__ unsigned long long redk[4];
    const int64_t r = blockIdx.x;
    const T *x = (const T *)a.logits + r * a.row_stride;
    auto add = [](float p, float q) { return p + q; };
    float m = -INFINITY;
    for (int v = threadIdx.x; v < a.vocab; v += 256) m = fmaxf(m, to_f32(x[v]));
    m = block_reduce(m, red, [](float p, float q) { return fmaxf(p, q); });
    const float ref = m == -INFINITY ? 0.f : m;
    float S = 0.f, W = 0.f;
    for (int v = threadIdx.x; v < a.vocab; v += 256) {
        const float d = to_f32(x[v]) - ref, e = expf(d);
        S += e;
        W += e * fmaxf(d, -1e4f);                                    // (a banned token: 0, not 0 * inf)
    }
    S = block_reduce(S, red, add);
    W = block_reduce(W, red, add);
    const bool none = S == 0.f;
    const float lse = none ? 0.f : ref + logf(S);
    if (threadIdx.x == 0) {
        if (a.entropy) a.entropy[r] = none ? 0.f : logf(S) - W / S;
        if (a.logprob) {
            const int t = a.tokens[r];
            a.logprob[r] = t < 0 ? 0.f : t >= a.vocab ? NAN : none ? -INFINITY : to_f32(x[t]) - lse;
        }
    }
    unsigned long long last = ~0ull;
    for (int i = 0; i < a.k; ++i) {
        unsigned long long best = 0;
        for (int v = threadIdx.x; v < a.vocab; v += 256) {
            const unsigned long long key = order_key(to_f32(x[v]), v);
            if (key < last && key > best) best = key;
        }
        best = block_reduce(best, redk, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
        if (threadIdx.x == 0) {
            a.top_logprob[r * a.k + i] = best ? key_value(best) - lse : -INFINITY;
            a.top_index[r * a.k + i] = best ? (int)(0xffffffffu - (unsigned)best) : -1;
        }
        last = best;
    }
}

} // namespace
} // namespace el

extern "C" int32_t el_attn_max_alternatives(void) { return el::kMaxAlternatives; }

extern "C" size_t el_attn_score_workspace_bytes(int32_t rows, int32_t vocab, int32_t k)
{
    if (rows < 1 || vocab < 1 || k < 0 || k > el::kMaxAlternatives) return 0;
    return 0;
}

extern "C" el_status el_attn_score_tokens(el_dtype dtype, const void *logits, int64_t row_stride, int32_t rows, int32_t vocab,
                                          const int32_t *tokens, float *logprob, float *entropy,
                                          int32_t k, float *top_logprob, int32_t *top_index,
                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (dtype != EL_F32 && dtype != EL_F16 && dtype != EL_BF16) return EL_ERR_UNSUPPORTED;
    if (!logits || rows < 1 || vocab < 1 || k < 0 || k > kMaxAlternatives) return EL_ERR_INVALID_ARG;
    if ((logprob && !tokens) || (k > 0 && (!top_logprob || !top_index))) return EL_ERR_INVALID_ARG;
    if ((rows > 1 && row_stride < vocab) || row_stride > ((int64_t)1 << 44)) return EL_ERR_INVALID_ARG;
    if ((uintptr_t)logits % dtype_size(dtype) != 0) return EL_ERR_INVALID_ARG;
    if (((uintptr_t)tokens | (uintptr_t)logprob | (uintptr_t)entropy | (uintptr_t)top_logprob | (uintptr_t)top_index) & 3) return EL_ERR_INVALID_ARG;
    const ScoreArgs a{(const char *)logits, row_stride, vocab, k, tokens, logprob, entropy, top_logprob, top_index};
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    if (dtype == EL_F32) hipLaunchKernelGGL((k_score_rows<float>), dim3(rows), dim3(256), 0, s, a);
    else if (dtype == EL_F16) hipLaunchKernelGGL((k_score_rows<f16_t>), dim3(rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_score_rows<bf16_t>), dim3(rows), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}
