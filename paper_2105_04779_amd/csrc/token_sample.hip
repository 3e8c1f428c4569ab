// The next token of a row of logits, drawn by a given random number from what temperature, top-k, top-p and min-p leave.
//
//   w_v = 2^43 exp((x_v - m) / T) as a 64-bit whole number, m the largest logit
//
// Sums of whole numbers are exact, so neither the order of a sum nor the split of a row changes which token is drawn.  All filters keep a beginning of one order (larger
// logits first, of equal ones the lowest index), so together they are a smallest logit, and how many of those equal to it stay.
#include <cfloat>
#include <cmath>
#include "mfma.h"

namespace el {
namespace {

constexpr int kLanes = 1024, kWaves = kLanes / 64;
constexpr int32_t kMaxVocab = 1 << 19;
constexpr unsigned long long kOne = 1ull << 43;                      // the largest logit's weight
constexpr double kLog2e = 1.4426950408889634074;

typedef unsigned long long u64;

struct SampleArgs {
    const char *logits;
    int64_t row_stride;                  // bytes
    int vocab;
    const float *uniform;
    el_attn_sample_rule rule;
    int32_t *tokens;
    float *logprob;
};

// What orders tokens: the value (-0 counts as 0), then the lower index.
__device__ __forceinline__ unsigned order32(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }
constexpr unsigned kNone = 0x007fffffu;                              // order of -inf: what may not follow is at or below it

// 2^y for y <= 0 as a whole number of 2^-43 (the series of e^(f ln 2) around the nearest whole exponent, f within a half: the first term left out is below 2^-47).
__device__ __forceinline__ u64 weight_of(double y)
{
    if (!(y > -44.0)) return y == y ? 0 : kOne;                      // (NaN: a difference of 0 times an infinite 1 / T)
    const double n = __builtin_rint(y), f = (y - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800.0;
    p = fma(p, f, 1.0 / 3628800.0);
    p = fma(p, f, 1.0 / 362880.0);
    p = fma(p, f, 1.0 / 40320.0);
    p = fma(p, f, 1.0 / 5040.0);
    p = fma(p, f, 1.0 / 720.0);
    p = fma(p, f, 1.0 / 120.0);
    p = fma(p, f, 1.0 / 24.0);
    p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    // (added to 2^52, the last bit of the sum is 1)
    return (u64)__double_as_longlong(ldexp(p, 43 + (int)n) + 0x1p52) & ((1ull << 52) - 1);
}

// Sums over the workgroup, the same in all lanes.
__device__ __forceinline__ u64 sum_all(u64 v)
{
    __shared__ u64 part[kWaves];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 s = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) s += part[i];
    return s;
}

// A row a workgroup.
template <typename T>
__global__ void __launch_bounds__(kLanes) k_sample(const SampleArgs a)
{
    __shared__ u64 bins[256];
    __shared__ unsigned found;
    __shared__ u64 above;
    __shared__ unsigned best;
    __shared__ int bad;
    __shared__ u64 sums[kLanes];
    __shared__ int ties[kLanes];
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x;
    const T *const row = (const T *)(a.logits + r * a.row_stride);
    const int V = a.vocab;
    if (tid == 0) { best = 0; bad = 0; }
    __syncthreads();
    unsigned mine = 0;
    bool wrong = false;
    for (int v = tid; v < V; v += kLanes) {
        const float x = to_f32(row[v]);
        wrong |= !(x < INFINITY);
        if (x > -INFINITY) mine = max(mine, order32(x));
    }
    if (wrong) bad = 1;
    atomicMax(&best, mine);
    __syncthreads();
    const unsigned top = best;
    if (bad || top <= kNone) {
        if (tid == 0) { a.tokens[r] = -1; if (a.logprob) a.logprob[r] = bad ? NAN : -INFINITY; }
        return;
    }
    const el_attn_sample_rule &f = a.rule;
    const float temperature = f.row_temperature ? f.row_temperature[r] : f.temperature;
    int k = f.row_top_k ? f.row_top_k[r] : f.top_k;
    const float top_p = f.row_top_p ? f.row_top_p[r] : f.top_p, min_p = f.row_min_p ? f.row_min_p[r] : f.min_p;
    if (!(temperature > 0.f) || min_p > 1.f || top_p <= 0.f) k = 1;
    const double m = (double)value_of(top), c = temperature > 0.f ? kLog2e / (double)temperature : 0.0;
    auto weight = [&](float x) { return weight_of(((double)x - m) * c); };

    // The order `least` at which a sum over all orders from the largest down reaches `target` (of counts, or of weights), and the sum above it.
    auto reach = [&](auto term, auto reached, unsigned floor_, u64 &over) {
        unsigned prefix = 0;
        over = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kLanes) bins[i] = 0;
            __syncthreads();
            for (int v = tid; v < V; v += kLanes) {
                const float x = to_f32(row[v]);
                const unsigned o = order32(x);
                if (o > kNone && o >= floor_ && (shift == 24 || o >> (shift + 8) == prefix >> (shift + 8))) atomicAdd(&bins[o >> shift & 255], term(x));
            }
            __syncthreads();
            if (tid == 0) {
                u64 s = over;
                int i = 255, last = -1;
                for (; i >= 0; --i) {
                    if (bins[i] == 0) continue;
                    last = i;
                    if (reached(s + bins[i])) break;
                    s += bins[i];
                }
                if (i < 0 && last >= 0) { i = last; s -= bins[last]; }           // (never reached: the smallest there is)
                found = prefix | (unsigned)max(i, 0) << shift;
                above = s;
            }
            __syncthreads();
            prefix = found; over = above;
            __syncthreads();
        }
        return prefix;
    };
    auto count_at = [&](unsigned o) {
        u64 n = 0;
        for (int v = tid; v < V; v += kLanes) n += order32(to_f32(row[v])) == o;
        return sum_all(n);
    };
    // what stays: orders above `least`, and the first `equal` tokens of that order
    unsigned least = kNone + 1;
    u64 equal = ~0ull;
    if (k > 0 && k < V) {
        u64 over;
        least = reach([](float) { return (u64)1; }, [&](u64 s) { return s >= (u64)k; }, 0u, over);
        equal = (u64)k - over;                                       // (fewer than k: more than there are)
    }
    auto total_of = [&]() {
        u64 w = 0;
        for (int v = tid; v < V; v += kLanes) {
            const float x = to_f32(row[v]);
            if (order32(x) > least) w += weight(x);
        }
        w = sum_all(w);
        w += min(equal, count_at(least)) * weight(value_of(least));
        return w;
    };
    if (top_p < 1.f && top_p > 0.f && k != 1) {
        const double want = (double)top_p * (double)total_of();
        u64 over;
        const unsigned o = reach([&](float x) { return weight(x); }, [&](u64 s) { return (double)s >= want; }, least, over);
        const u64 w = weight(value_of(o));
        // those of this order that have less than `want` before them
        u64 n = w ? (u64)ceil(fmax(want - (double)over, 0.0) / (double)w) : 1;
        if (n > 0 && !((double)(over + (n - 1) * w) < want)) --n;
        if ((double)(over + n * w) < want) ++n;
        n = max(n, (u64)1);
        if (o == least) equal = min(equal, n);
        else { least = o; equal = n; }
    }
    const double low = min_p > 0.f && min_p <= 1.f ? (double)min_p * (double)kOne : 0.0;
    auto kept = [&](float x) { return (double)weight(x) >= low; };

    // a segment of the vocabulary a lane: weights above `least`, and how many equal it
    auto segment = [&](int from, int to, u64 &w, int &n) {
        w = 0; n = 0;
        for (int v = from; v < to; ++v) {
            const float x = to_f32(row[v]);
            const unsigned o = order32(x);
            if (o > least && kept(x)) w += weight(x);
            n += o == least && kept(x);
        }
    };
    const u64 w_least = weight(value_of(least));
    const int each = (V + kLanes - 1) / kLanes;
    segment(min(tid * each, V), min((tid + 1) * each, V), sums[tid], ties[tid]);
    __syncthreads();
    if (tid == 0) {
        u64 total = 0, left = equal;
        for (int i = 0; i < kLanes; ++i) { const u64 n = min(left, (u64)ties[i]); left -= n; total += sums[i] + n * w_least; }
        const double target = (double)a.uniform[r] * (double)total;
        u64 upto = 0;
        left = equal;
        int chosen = -1;
        u64 w_chosen = 0;
        for (int i = 0; i < kLanes; ++i) {
            const u64 n = min(left, (u64)ties[i]), w = sums[i] + n * w_least;
            if (w > 0 && ((double)(upto + w) > target || upto + w == total)) {
                for (int v = i * each; v < min((i + 1) * each, V); ++v) {
                    const float x = to_f32(row[v]);
                    const unsigned o = order32(x);
                    const bool there = kept(x) && (o > least || (o == least && left > 0));
                    if (!there) continue;
                    if (o == least) --left;
                    const u64 wx = weight(x);
                    if (wx == 0) continue;
                    chosen = v; w_chosen = wx;
                    upto += wx;
                    if ((double)upto > target) break;
                }
                break;
            }
            left -= n;
            upto += w;
        }
        a.tokens[r] = chosen;
        if (a.logprob) a.logprob[r] = (float)log((double)w_chosen / (double)total);
    }
}

} // namespace
} // namespace el

extern "C" size_t el_attn_sample_workspace_bytes(el_dtype dtype, int32_t rows, int32_t vocab) { (void)dtype; (void)rows; (void)vocab; return 0; }

extern "C" el_status el_attn_sample_tokens(el_dtype dtype, const void *logits, int64_t row_stride, int32_t rows, int32_t vocab, const float *uniform,
                                           const el_attn_sample_rule *rule, int32_t *tokens, float *logprob,
                                           void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (dtype != EL_F32 && dtype != EL_F16 && dtype != EL_BF16) return EL_ERR_UNSUPPORTED;
    if (!logits || !uniform || !rule || !tokens || rows < 1 || rows > 1 << 23 || vocab < 1) return EL_ERR_INVALID_ARG;
    if (vocab > kMaxVocab) return EL_ERR_UNSUPPORTED;
    const int64_t es = (int64_t)dtype_size(dtype);
    if ((rows > 1 && row_stride < vocab) || row_stride > ((int64_t)1 << 44) || out_of_reach(rows, row_stride * es) || (uintptr_t)logits % es) return EL_ERR_INVALID_ARG;
    if (((uintptr_t)uniform | (uintptr_t)tokens | (uintptr_t)logprob | (uintptr_t)rule->row_temperature | (uintptr_t)rule->row_top_k |
         (uintptr_t)rule->row_top_p | (uintptr_t)rule->row_min_p) & 3) return EL_ERR_INVALID_ARG;
    if (!rule->row_temperature && !(rule->temperature >= 0.f && rule->temperature < INFINITY)) return EL_ERR_INVALID_ARG;
    (void)workspace; (void)workspace_bytes;
    const SampleArgs a{(const char *)logits, row_stride * es, vocab, uniform, *rule, tokens, logprob};
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    if (dtype == EL_F32) hipLaunchKernelGGL((k_sample<float>), dim3(rows), dim3(kLanes), 0, s, a);
    else if (dtype == EL_F16) hipLaunchKernelGGL((k_sample<f16_t>), dim3(rows), dim3(kLanes), 0, s, a);
    else hipLaunchKernelGGL((k_sample<bf16_t>), dim3(rows), dim3(kLanes), 0, s, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}
