// The next token of a row of logits, drawn by a given random number from what temperature, top-k, top-p and min-p leave.
//
//   w_v = 2^43 exp((x_v - m) / T) as a 64-bit whole number, m the largest logit
//
// Sums of whole numbers are exact, so neither the order of a sum nor the split of a row changes which token is drawn, and sums in LDS may be atomic.  All filters
// keep a beginning of one order (larger logits first, of equal ones the lowest index), so together they are a smallest logit, `least`, and how many of those equal
// to it stay, `equal`.
//
// A row a workgroup of 16 wavefronts, each with a sixteenth of it (8 with an eighth where the rows are more than the compute units).  Few tokens (top-k): those not below a bound from the lanes' maxima are collected and ranked by counting.
// Otherwise the bound of top-p or top-k is found by a histogram of weights (or counts) over 512 ranges of logits, one for each wavefront, and the tokens of the
// range that it falls into are ranked; a range of too many is cut into 512 again.  The sums of the ranges above are then each wavefront's share of what is left, so
// the token's share is known without another look at the row, and only that is gone through in order.
//
// Bound by the vector ALU, 23 operations a logit for its weight, 16 of them of 64 bits (HBM alone would allow a row in 11 us on each compute unit), and for rows in
// fp32 as much by HBM, from which they come 2.6 times: 688 MB in 140 to 150 us for 512 of 128003.  us of a row in
// bf16, one on each compute unit, 128003 logits: maxima 11 (HBM's rate), all weights 30, or 43 with their histogram (the rest is atomics in LDS, 11 to 18 clocks
// each), tokens of the range 17, ranked 5, the share and the token 6.  256 rows with settings of their own 80 (97 when rows with top-p and min-p were
// always cut by the one before the other), 4 rows of 50265 with top-k 50 and all filters 17, three looks at the row.
// More rows than compute units: workgroups of 512 lanes, two of which share one, so that a row computes while the other waits.  us with 1024 / 512: 512 rows of 128003 in bf16,
// top-p 0.9 170 / 157, top-k 40 70 / 59, nothing 100 / 101; of 32000, top-p 72 / 53; 2000 of 32000, top-k and top-p of their own 182 / 123.  Rows that take longer are
// begun first: 512 in fp32, half of them with top-p, 178 in their order (176 with 512 lanes), 160 (three passes a captured graph; 133 to 154 among others, by the rows' luck).
#include <cfloat>
#include <cmath>
#include <type_traits>
#include "mfma.h"

namespace el {
namespace {

constexpr int kBins = 512;
constexpr int kEach = 512;               // tokens that a wavefront collects
constexpr int kComputeUnits = 256;
constexpr int kRowsOfLaunch = 1 << 22;   // a launch has fewer than 2^32 lanes
constexpr int kOrdered = 4096;           // rows up to which those that take longer are begun first
constexpr int kFewTokens = 128;          // top-k up to which the bound from the lanes' maxima is used
constexpr int32_t kMaxVocab = 1 << 19;
constexpr double kLog2e = 1.4426950408889634074;

typedef unsigned long long u64;
__device__ __forceinline__ u64 lesser(u64 x, u64 y) { return x < y ? x : y; }
constexpr u64 kOne = 1ull << 43;         // the largest logit's weight

// What orders tokens: the value (-0 counts as 0), then the lower index.
__device__ __forceinline__ unsigned order32(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }
constexpr unsigned kLowest = 0x00800000u;                            // order of the lowest number: -inf lies below
__device__ __forceinline__ u64 key_of(unsigned order, int v) { return ((u64)order << 32) | (0xffffffffu - (unsigned)v); }

// 2^f for |f| <= 1/2 is 1 + f q(f): q the interpolation of (2^f - 1) / f at the nine Chebyshev nodes, off by 2^-44.6 of the result at most.  (In kernel arguments: a
// product's addend comes from a scalar register then, where a constant is moved into a vector one for every use.)
struct Powers { double q[9]; };
constexpr Powers kPowers{{0x1.b63880d302e52p-24, 0x1.63d13636a87f6p-20, 0x1.ffcb95157f403p-17, 0x1.4308ac85aa333p-13, 0x1.5d87fe86fe90ep-10, 0x1.3b2ab7181b75ap-7,
                          0x1.c6b08d7047e52p-5, 0x1.ebfbdff823cedp-3, 0x1.62e42fefa39efp-1}};

struct SampleArgs {
    const char *logits;
    int64_t row_stride;                  // bytes
    int vocab;
    const float *uniform;
    el_attn_sample_rule rule;
    int32_t *tokens;
    float *logprob;
    Powers powers;
    int rows;
    bool by_cost;                        // rows that take longer first
};

// Does row r need the sums over ranges?
__device__ __forceinline__ bool takes_longer(const SampleArgs &a, int r)
{
    const el_attn_sample_rule &f = a.rule;
    const int k = f.row_top_k ? f.row_top_k[r] : f.top_k;
    const float p = f.row_top_p ? f.row_top_p[r] : f.top_p;
    const bool counted = k > 0 && k < a.vocab;
    return counted ? k > kFewTokens : p > 0.f && p < 1.f;
}

// The weights of a row: exp((x - m) / T) in units of 2^-43, whole numbers, without a branch.
struct Weight {
    static constexpr u64 kBase = 0x4330000000000000ull;              // the bits of 2^52
    const Powers &p;
    double c, md, low;                   // log2(e) / T, m; a logit down to `low` weighs 2^-45: nothing
    __device__ __forceinline__ Weight(const Powers &powers, float m, float temperature) : p(powers), md((double)m)
    {
        // (`low` below m as a number of 64 bits: at 2^-30 of m the next smaller logit weighs nothing either way)
        c = fmin(fmax(kLog2e / (double)temperature, 1e-300), 45.0 * 0x1p30 / fmax(fabs(md), 1e-300));
        low = md - 45.0 / c;
    }
    // behind the bits of 2^52
    __device__ __forceinline__ u64 raw(float x) const
    {
        constexpr double kRound = 0x1.8p52 + 43.0;                   // (a sum's last bits are the whole exponent, plus 43)
        const double d = fmax((double)x, low) - md, t = fma(d, c, kRound), f = fma(d, c, kRound - t);
        double v = p.q[0];
#pragma unroll
        for (int i = 1; i < 9; ++i) v = fma(v, f, p.q[i]);
        v = fma(v, f, 1.0);
        const u64 b = (u64)__double_as_longlong(v) + ((u64)__double_as_longlong(t) << 52);
        return (u64)__double_as_longlong(__longlong_as_double((long long)b) + 0x1p52);
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kBase; }
};

// Eight logits, which lie at a 16-byte boundary.
template <typename T> struct Eight {
    static constexpr int W = sizeof(T) / 2;                          // pieces of 16 bytes
    u4 w[W];
    __device__ __forceinline__ static Eight of(const T *at, bool there)
    {
        // (all -inf where there is none)
        constexpr unsigned none = std::is_same<T, float>::value ? 0xff800000u : std::is_same<T, bf16_t>::value ? 0xff80ff80u : 0xfc00fc00u;
        Eight e;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            e.w[i] = u4{none, none, none, none};
            if (there) e.w[i] = ((const u4 *)at)[i];
        }
        return e;
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (std::is_same<T, float>::value) return __uint_as_float(w[i >> 2][i & 3]);
        const unsigned u = w[0][i >> 1];             // (a bit cast of a vector's element itself takes element 0 whatever the index: through a copy)
        if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
        else return (float)__builtin_bit_cast(h2, u)[i & 1];
    }
};

// What a workgroup of LANES lanes does with a row.
template <int LANES> struct Sampling {
static constexpr int kLanes = LANES, kWaves = kLanes / 64;
static constexpr int kList = kWaves > 8 ? 4096 : (kWaves - 1) * kBins;       // tokens that are collected, of all wavefronts
static constexpr int kRanked = kLanes;           // of them, those that are ranked by counting: one a lane

// A row: `full` pieces of 8 logits behind `head` of them, `per` of them a wavefront's; the first wavefront has the elements before the pieces, the last those
// behind them, so shares lie one behind the other.
template <typename T> struct Row {
    static constexpr int N = 8;
    const T *row;
    int head, full, per, vocab;
    __device__ __forceinline__ Row(const SampleArgs &a, int64_t r)
    {
        row = (const T *)(a.logits + r * a.row_stride);
        vocab = a.vocab;
        head = min((int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T), vocab);
        full = (vocab - head) / N;
        per = max((full + kWaves - 1) / kWaves, 1);
    }
    __device__ __forceinline__ int share_of(int v) const { return v < head ? 0 : v >= head + full * N ? kWaves - 1 : (v - head) / N / per; }
    // g(x, index of the first) for N neighbours of wavefront w's share at a time, -inf where there is none in the row
    template <typename G> __device__ __forceinline__ void pieces(int w, G g) const
    {
        constexpr int AHEAD = std::is_same<T, float>::value ? 3 : 4;                 // under way; one copy of g, whose code would else fill the instruction cache
        const int lane = threadIdx.x & 63, end = min((w + 1) * per, full);
        const T *const from = row + head;
        Eight<T> v[AHEAD];
        int p = w * per + lane;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) v[j] = Eight<T>::of(from + (int64_t)(p + 64 * j) * N, p + 64 * j < end);
#pragma unroll 1
        for (int q = w * per; q < end; q += 64, p += 64) {
            const Eight<T> now = v[0];
#pragma unroll
            for (int j = 0; j + 1 < AHEAD; ++j) v[j] = v[j + 1];
            v[AHEAD - 1] = Eight<T>::of(from + (int64_t)(p + 64 * AHEAD) * N, p + 64 * AHEAD < end);
            float x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = now.at(i);
            g(x, head + p * N);
        }
        if (w == 0 || w == kWaves - 1) {
            const int v = w == 0 ? lane : head + full * N + lane, stop = w == 0 ? head : vocab;
            float x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = -INFINITY;
            if (v < stop) x[0] = to_f32(row[v]);
            g(x, v);
        }
    }
    __device__ __forceinline__ int begin_piece(int w) const { return min(w * per, full); }
    // f(x, index), one after the other
    template <typename F> __device__ __forceinline__ void each(int w, F f) const
    {
        pieces(w, [&](const float (&x)[N], int v) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) f(x[i], v + i);
        });
    }
};

struct Shared {
    u64 bins[kWaves][kBins];
    u64 list[kList + 8];
    int found_n[kWaves];
    u64 part[kWaves];
    u64 wave_sum[kWaves];                // weights left in each share, above `least`
    int wave_ties[kWaves];               // tokens of the order `least`
    unsigned best[256];
    float part_m[kWaves];
    unsigned lowest, highest;
    int count, bad, token, cross;
    u64 before;
    // (what a wavefront collects lies where its ranges were, which have been added up by then)
    __device__ __forceinline__ u64 *found(int w) { return bins[w]; }
    // (the ranked list lies where the last wavefronts' ranges were, which have been added up by then)
    __device__ __forceinline__ u64 *sorted() { return bins[kWaves - 2]; }
};
static_assert(2 * kBins >= kRanked && kBins >= kEach && (kWaves - 1) * kBins >= kList && kLanes >= kBins, "room of the lists");

// Sum over the lanes before this one in the workgroup; `total`: of all.
static __device__ __forceinline__ u64 sum_before(Shared &s, u64 v, u64 &total)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    u64 up = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const u64 x = __shfl_up(up, o, 64); if (lane >= o) up += x; }
    __syncthreads();
    if (lane == 63) s.part[w] = up;
    __syncthreads();
    u64 first = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) { if (i < w) first += s.part[i]; total += s.part[i]; }
    return first + up - v;
}
static __device__ __forceinline__ u64 sum_wave(u64 v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// The first of the orders from `from` to `to` whose number is `in`, as all behind it are, the last one among them: 64 candidates a round.
template <typename F> static __device__ __forceinline__ unsigned first_order(unsigned from, unsigned to, F in)
{
    const unsigned lane = threadIdx.x & 63;
    unsigned size = to - from;                                       // the answer lies in [from, from + size]
    while (size) {
        const unsigned step = size / 64 + 1;
        const u64 there = __ballot(in(value_of(from + min(step * lane, size))));
        const unsigned i = there ? (unsigned)__ffsll((long long)there) - 1 : 64;
        const unsigned upper = i < 64 ? min(step * i, size) : size, lower = i == 0 ? 0 : min(step * (i - 1), size) + 1;
        from += lower;
        size = upper - lower;
    }
    return from;
}

// The k-th largest of 256 numbers, four a lane, without its bits below 16 (0: fewer than k are above 0).
static __device__ __forceinline__ unsigned kth_of(const unsigned (&mine)[4], int k)
{
    unsigned bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const unsigned t = bound | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += __popcll(__ballot(mine[i] >= t));
        if (n >= k) bound = t;
    }
    return bound;
}

// A wavefront's own list: those that it takes, one behind the other.
struct Taken {
    u64 *const to;
    int n = 0;
    unsigned lowest = 0xffffffffu, highest = 0;
    __device__ __forceinline__ void take(bool here, unsigned o, int v)
    {
        const u64 mask = __builtin_amdgcn_ballot_w64(here);
        if (!mask) return;
        const int at = n + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
        if (here) {
            if (at < kEach) to[at] = key_of(o, v);
            lowest = min(lowest, o); highest = max(highest, o);
        }
        n += __popcll(mask);
    }
};
// The wavefronts' lists as one: how many, or more than kList if there is not room for all.  All lanes.
static __device__ __forceinline__ int gather(Shared &s, const Taken &t)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    __syncthreads();
    if (lane == 0) s.found_n[w] = t.n;
    __syncthreads();
    int first = 0, all = 0, most = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) { const int n = s.found_n[i]; if (i < w) first += n; all += n; most = max(most, n); }
    if (most > kEach || all > kList) return max(all, kList + 1);
    for (int i = lane; i < t.n; i += 64) s.list[first + i] = t.to[i];
    __syncthreads();
    return all;
}

// The list's n keys (followed by zeros) in descending order.  All lanes; n up to kRanked.
static __device__ __forceinline__ void rank_list(Shared &s, int n)
{
    const int tid = threadIdx.x;
    if (tid < 8) s.list[n + tid] = 0;
    __syncthreads();
    if (tid < n) {
        const u64 key = s.list[tid];
        int rank = 0;
        for (int o = 0; o < n; o += 8) {
            u64 other[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = s.list[o + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) rank += other[i] > key;
        }
        s.sorted()[rank] = key;
    }
    __syncthreads();
}

template <typename T>
static __device__ __forceinline__ void run(const SampleArgs &a)
{
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int64_t r = blockIdx.x;
    if (a.by_cost) {
        const int each = (a.rows + kLanes - 1) / kLanes, first = min(tid * each, a.rows), last = min(first + each, a.rows);
        u64 longer = 0, all;
        for (int i = first; i < last; ++i) longer += takes_longer(a, i);
        const u64 before = sum_before(s, longer, all), mine = blockIdx.x;
        const bool want = mine < all;
        const u64 front = want ? before : all + (u64)first - before, here = want ? longer : (u64)(last - first) - longer;
        if (mine >= front && mine < front + here) {
            int i = first;
            for (u64 n = mine - front;; ++i) if (takes_longer(a, i) == want && n-- == 0) break;
            s.cross = i;
        }
        __syncthreads();
        r = __builtin_amdgcn_readfirstlane(s.cross);
    }
    const Row<T> row(a, r);

    // ---- the largest logit, and the lanes' maxima, four lanes each ----
    float m = -INFINITY;
    bool wrong = false;
    row.each(w, [&](float x, int) { m = fmaxf(m, x); wrong |= !(x < INFINITY); });
    if (tid == 0) { s.bad = 0; s.token = 0x7fffffff; }
    {
        float m4 = fmaxf(m, quad_xor1(m));
        if constexpr (kLanes == 1024) m4 = fmaxf(m4, quad_xor2(m4));
        constexpr int SHARE = kLanes / 256;
        if (tid % SHARE == 0) s.best[tid / SHARE] = m4 > -INFINITY ? order32(m4) : 0u;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        if (lane == 0) s.part_m[w] = m;
    }
    const el_attn_sample_rule &f = a.rule;
    const float temperature = f.row_temperature ? f.row_temperature[r] : f.temperature;
    int k = f.row_top_k ? f.row_top_k[r] : f.top_k;
    const float top_p = f.row_top_p ? f.row_top_p[r] : f.top_p, min_p = f.row_min_p ? f.row_min_p[r] : f.min_p, uniform = a.uniform[r];
    __syncthreads();
    if (wrong) s.bad = 1;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = fmaxf(m, s.part_m[i]);
    __syncthreads();
    if (s.bad || m == -INFINITY) {
        if (tid == 0) { a.tokens[r] = -1; if (a.logprob) a.logprob[r] = s.bad ? NAN : -INFINITY; }
        return;
    }
    if (!(temperature > 0.f) || min_p > 1.f || top_p <= 0.f || k == 1) {
        // the first in order
        int first = 0x7fffffff;
        row.each(w, [&](float x, int v) { if (x == m) first = min(first, v); });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
        if (lane == 0) atomicMin(&s.token, first);
        __syncthreads();
        if (tid == 0) { a.tokens[r] = s.token; if (a.logprob) a.logprob[r] = 0.f; }
        return;
    }
    const Weight weight(a.powers, m, temperature);
    const double low = min_p > 0.f ? (double)min_p * (double)kOne : 0.0;                 // weights that min-p leaves
    // (from the logit: an unlikely token's weight is few units, which its logarithm would show.  The total is 1 or more and off by 2^-44 a token)
    auto write = [&](int v, float x, u64 total) {
        a.tokens[r] = v;
        if (a.logprob) a.logprob[r] = (float)(((double)x - (double)m) / (double)temperature - log((double)total * (1.0 / (double)kOne)));
    };
    const bool by_count = k > 0 && k < row.vocab, by_weight = top_p < 1.f;

    if (by_count && k <= kFewTokens) {
        const unsigned maxima[4] = {s.best[lane], s.best[lane + 64], s.best[lane + 128], s.best[lane + 192]};
        const unsigned bound = kth_of(maxima, k);
        const float least = bound ? value_of(bound) : -FLT_MAX;
        Taken t{s.found(w)};
        row.each(w, [&](float x, int v) __attribute__((always_inline)) { t.take(x >= least, order32(x), v); });
        const int n = gather(s, t);
        if (n <= kRanked) {
            rank_list(s, n);
            // a token a lane, in order; few enough that each lane adds up what it needs
            const bool mine = tid < min(n, k);
            const u64 key = mine ? s.sorted()[tid] : 0;
            const u64 wv = mine ? weight(value_of((unsigned)(key >> 32))) : 0;
            u64 total;
            const u64 before = sum_before(s, wv, total);
            const bool kept = mine && (tid == 0 || ((!by_weight || (double)before < (double)top_p * (double)total) && (double)wv >= low));
            // (the kept are a beginning: weights do not grow)
            u64 left;
            (void)sum_before(s, kept ? wv : 0, left);
            const double target = uniform < 0.f ? 0.0 : (double)uniform * (double)left;
            const int v = (int)(0xffffffffu - (unsigned)key);
            if (tid < kFewTokens) { s.bins[0][tid] = kept ? wv : 0; s.bins[1][tid] = (u64)v; }
            if (tid == 0) s.cross = -1;
            __syncthreads();
            u64 upto = 0;
            if (kept && wv)
                for (int i = 0; i < min(n, k); ++i) upto += (int)s.bins[1][i] <= v ? s.bins[0][i] : 0;
            if (kept && wv) {
                if ((double)upto > target) atomicMin(&s.token, v);
                if (upto == left) s.cross = v;                       // the last in the order of the vocabulary
            }
            __syncthreads();
            const int chosen = s.token != 0x7fffffff ? s.token : s.cross;
            if (kept && wv && v == chosen) write(v, value_of((unsigned)(key >> 32)), left);
            return;
        }
        __syncthreads();
    }

    // What is left: logits above `least`, and the first `equal` tokens of those equal to it.
    float least = -INFINITY;
    u64 equal = 0;
    bool sums = false;                                               // wave_sum and wave_ties are those of (least, equal)
    unsigned min_from = 0;                                           // the smallest order that min-p leaves
    // Sets them to where a sum in order, of weights or (COUNT) of ones, reaches a bound: `reached(sum)`.  begin(total) is told the sum of all; false ends it.  So does
    // min-p where it ends in a range before: the tokens that the bound falls between are not looked for then.
    auto select = [&](auto is_count, auto begin, auto reached, float steps) {
        constexpr bool COUNT = decltype(is_count)::value;
        // (those equal to `least` take part as well: of them, the lowest there are, no more than `equal` are taken in the end)
        const float floor_ = fmaxf(least, -FLT_MAX);
        auto term = [&](float x) __attribute__((always_inline)) { if constexpr (COUNT) return (u64)1; else return weight(x); };
        auto bin_of = [&](float x) __attribute__((always_inline)) { return (int)fminf((m - x) * steps, (float)(kBins - 1)); };      // (does not fall where logits do)
        // of n equal tokens of weight t, behind a sum of `before`, the fewest that reach the bound
        auto fewest = [&](u64 before, u64 t, int n) {
            int a1 = 1, b1 = n;
            while (a1 < b1) { const int mid = (a1 + b1) / 2; if (reached(before + mid * t)) b1 = mid; else a1 = mid + 1; }
            return (u64)a1;
        };
        u64 over = 0;
        unsigned lo = 0, hi = 0, width = 0;                          // from the second round on: ranges of orders
        if (tid < kWaves) { s.wave_sum[tid] = 0; s.wave_ties[tid] = 0; }
        for (bool first = true;; first = false) {
            for (int i = tid; i < kWaves * kBins; i += kLanes) (&s.bins[0][0])[i] = 0;
            if (tid == 0) { s.lowest = 0xffffffffu; s.highest = 0; }
            __syncthreads();
            u64 *const bins = s.bins[w];
            if (first) {
                // (the last range, which may hold most of a row, is summed in registers)
                u64 last = 0;
                row.pieces(w, [&](const float (&x)[Row<T>::N], int) __attribute__((always_inline)) {
                    constexpr int AT_ONCE = 4;       // (more weights side by side do not fit the registers)
#pragma unroll
                    for (int i0 = 0; i0 < Row<T>::N; i0 += AT_ONCE) {
                        u64 t[AT_ONCE];
#pragma unroll
                        for (int i = 0; i < AT_ONCE; ++i) t[i] = term(x[i0 + i]);
#pragma unroll
                        for (int i = 0; i < AT_ONCE; ++i) {
                            const int bin = bin_of(x[i0 + i]);
                            const bool in = x[i0 + i] >= floor_;
                            if (in && bin < kBins - 1) atomicAdd(&bins[bin], t[i]);
                            last += in && bin == kBins - 1 ? t[i] : 0;
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
                last = sum_wave(last);
                if (lane == 0) bins[kBins - 1] = last;
            } else {
                row.each(w, [&](float x, int) __attribute__((always_inline)) {
                    const unsigned o = order32(x);
                    if (o >= lo && o <= hi) atomicAdd(&bins[(hi - o) / width], term(x));
                });
            }
            __syncthreads();
            u64 mine = 0, total;
            if (tid < kBins)
                for (int i = 0; i < kWaves; ++i) mine += s.bins[i][tid];
            const u64 before = over + sum_before(s, mine, total);
            if (first && !begin(total)) return;
            if (tid < kBins && mine && reached(before + mine) && !reached(before)) { s.cross = tid; s.before = before; }
            __syncthreads();
            const int cross = s.cross;
            over = s.before;
            if (!COUNT && first && min_from && bin_of(value_of(min_from)) < cross) return;
            u64 share = 0;
            for (int i = lane; i < cross; i += 64) share += bins[i];
            share = sum_wave(share);
            if (lane == 0) s.wave_sum[w] += share;
            // the tokens of that range
            Taken found{s.found(w)};
            if (first) {
                // (the range's own bounds: two comparisons a logit)
                const unsigned top = order32(m), from = first_order(order32(floor_), top, [&](float x) { return bin_of(x) <= cross; });
                const unsigned to = cross ? first_order(from, top, [&](float x) { return bin_of(x) < cross; }) - 1 : top;
                const float x_lo = value_of(from), x_hi = value_of(to);
                row.each(w, [&](float x, int v) __attribute__((always_inline)) { found.take(x >= x_lo && x <= x_hi, order32(x), v); });
            } else {
                row.each(w, [&](float x, int v) __attribute__((always_inline)) {
                    const unsigned o = order32(x);
                    found.take(o >= lo && o <= hi && (int)((hi - o) / width) == cross, o, v);
                });
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                found.lowest = min(found.lowest, (unsigned)__shfl_xor((int)found.lowest, o, 64));
                found.highest = max(found.highest, (unsigned)__shfl_xor((int)found.highest, o, 64));
            }
            if (lane == 0) { atomicMin(&s.lowest, found.lowest); atomicMax(&s.highest, found.highest); }
            const int n = gather(s, found);
            lo = s.lowest; hi = s.highest;
            __syncthreads();
            if (n > kList && lo != hi) { width = (hi - lo) / kBins + 1; continue; }
            float last;
            u64 taken;
            if (lo == hi) {
                // all equal: the fewest that reach it
                last = value_of(lo);
                taken = fewest(over, term(last), n);
                if (n > kList) {
                    int ties = 0;
                    row.each(w, [&](float x, int) { ties += x == last; });
                    ties = (int)sum_wave(ties);
                    if (lane == 0) s.wave_ties[w] = ties;
                } else {
                    for (int i = tid; i < n; i += kLanes) atomicAdd(&s.wave_ties[row.share_of((int)(0xffffffffu - (unsigned)s.list[i]))], 1);
                }
            } else {
                // 512 ranges of orders, until that which the bound falls into holds one order, or few tokens, which are looked at one by one
                constexpr int kFew = 64;
                auto order_of = [&](int i) { return (unsigned)(s.list[i] >> 32); };
                u64 *const ranges = s.bins[0], *const few = s.bins[1];           // few: keys
                for (;;) {
                    const unsigned step = (hi - lo) / kBins + 1;
                    if (tid < kBins) ranges[tid] = 0;
                    if (tid == 0) { s.count = 0; s.lowest = 0xffffffffu; s.highest = 0; }
                    __syncthreads();
                    for (int i = tid; i < n; i += kLanes) {
                        const unsigned o = order_of(i);
                        if (o >= lo && o <= hi) atomicAdd(&ranges[(hi - o) / step], term(value_of(o)));
                    }
                    __syncthreads();
                    const u64 here = tid < kBins ? ranges[tid] : 0;
                    u64 all;
                    const u64 upto = over + sum_before(s, here, all);
                    if (here && reached(upto + here) && !reached(upto)) { s.cross = tid; s.before = upto; }
                    __syncthreads();
                    const unsigned range = (unsigned)s.cross;
                    over = s.before;
                    for (int i = tid; i < n; i += kLanes) {
                        const unsigned o = order_of(i);
                        if (o < lo || o > hi || (hi - o) / step != range) continue;
                        few[atomicAdd(&s.count, 1)] = s.list[i];
                        atomicMin(&s.lowest, o); atomicMax(&s.highest, o);
                    }
                    __syncthreads();
                    lo = s.lowest; hi = s.highest;
                    if (lo == hi || s.count <= kFew) break;
                    __syncthreads();
                }
                const int few_n = s.count;
                __syncthreads();
                if (lo == hi) {
                    last = value_of(lo);
                    taken = fewest(over, term(last), few_n);
                } else {
                    if (tid == 0) { s.lowest = 0xffffffffu; s.count = 0; }
                    __syncthreads();
                    bool kept = false;
                    if (tid < few_n) {
                        u64 first = over;
                        for (int i = 0; i < few_n; ++i) first += few[i] > few[tid] ? term(value_of((unsigned)(few[i] >> 32))) : 0;
                        kept = !reached(first);
                        if (kept) atomicMin(&s.lowest, (unsigned)(few[tid] >> 32));
                    }
                    __syncthreads();
                    const unsigned last_o = s.lowest;
                    last = value_of(last_o);
                    if (kept && (unsigned)(few[tid] >> 32) == last_o) atomicAdd(&s.count, 1);
                    __syncthreads();
                    taken = (u64)s.count;
                }
                for (int i = tid; i < n; i += kLanes) {
                    const u64 key = s.list[i];
                    const float x = value_of((unsigned)(key >> 32));
                    const int at = row.share_of((int)(0xffffffffu - (unsigned)key));
                    if (x > last) atomicAdd(&s.wave_sum[at], term(x));
                    if (x == last) atomicAdd(&s.wave_ties[at], 1);
                }
            }
            equal = last == least ? lesser(equal, taken) : taken;
            least = last;
            sums = !COUNT;
            __syncthreads();
            return;
        }
    };
    u64 dropped = 0;                                                 // of the tokens equal to `least`, those that top-k does not leave
    if (by_count) {
        select(std::true_type{}, [&](u64 total) { return total > (u64)k; }, [&](u64 sum) { return sum >= (u64)k; }, 16.f);
        if (equal) {
            for (int i = 0; i < kWaves; ++i) dropped += s.wave_ties[i];
            dropped -= equal;
        }
        __syncthreads();
    }
    if (low > 0.0) min_from = first_order(max(order32(least), kLowest), order32(m), [&](float x) { return (double)weight(x) >= low; });
    if (by_weight) {
        double bound = 0.0;
        const u64 less = dropped ? dropped * weight(least) : 0;
        select(std::false_type{}, [&](u64 total) { bound = (double)top_p * (double)(total - less); return true; }, [&](u64 sum) { return (double)sum >= bound; },
               (float)fmin(weight.c * (kBins / 24.0), 1e30));          // (what weighs less than 2^-24 is one range)
    }
    if (min_from > max(order32(least), kLowest)) { least = value_of(min_from - 1); equal = 0; sums = false; }
    const u64 w_least = equal ? weight(least) : 0;
    if (!sums) {
        u64 sum = 0;
        row.pieces(w, [&](const float (&x)[Row<T>::N], int) __attribute__((always_inline)) {
            float most = x[0];
#pragma unroll
            for (int i = 1; i < Row<T>::N; ++i) most = fmaxf(most, x[i]);
            if (!__builtin_amdgcn_ballot_w64(most > least)) return;
#pragma unroll
            for (int i = 0; i < Row<T>::N; ++i) {
                sum += weight(x[i] > least ? x[i] : -INFINITY);
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        });
        sum = sum_wave(sum);
        int ties = 0;
        if (equal) row.each(w, [&](float x, int) __attribute__((always_inline)) { ties += x == least; });
        ties = (int)sum_wave(ties);
        if (lane == 0) { s.wave_sum[w] = sum; s.wave_ties[w] = ties; }
        __syncthreads();
    }

    // ---- the share that the token lies in, then the token ----
    auto ties_left = [&](u64 before, int n) { return before >= equal ? 0ull : lesser(equal - before, (u64)n); };
    // (a share a lane; sums over the lanes up to it)
    auto upto = [&](u64 v) {
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) { const u64 x = __shfl_up(v, o, 64); if (lane >= o) v += x; }
        return v;
    };
    const int ties_here = lane < kWaves ? s.wave_ties[lane] : 0;
    const u64 ties_before = upto((u64)ties_here) - ties_here, here = lane < kWaves ? s.wave_sum[lane] + ties_left(ties_before, ties_here) * w_least : 0;
    const u64 sum_upto = upto(here), total = __shfl(sum_upto, kWaves - 1, 64);
    const double target = uniform < 0.f ? 0.0 : (double)uniform * (double)total;
    const u64 in = __ballot(lane < kWaves && here && ((double)sum_upto > target || sum_upto == total));
    const int share = __ffsll((long long)in) - 1;                    // (some: the largest logit is left)
    u64 base = __shfl(sum_upto - here, share, 64), base_ties = __shfl(ties_before, share, 64);
    // a lane takes pieces of the share one behind the other; the elements before the first piece of the row are lane 0's too, those behind the last one the last lane's
    constexpr int N = Row<T>::N;
    const int p_begin = row.begin_piece(share), p_end = share == kWaves - 1 ? row.full : row.begin_piece(share + 1), each = (p_end - p_begin + kLanes - 1) / kLanes;
    const int p0 = min(p_begin + tid * each, p_end), p1 = min(p0 + each, p_end);
    const bool has_head = share == 0 && tid == 0, has_tail = share == kWaves - 1 && tid == kLanes - 1;
    auto walk = [&](auto f) __attribute__((always_inline)) {         // f(x, index) in order, until it returns true
        if (has_head)
            for (int v = 0; v < row.head; ++v) if (f(to_f32(row.row[v]), v)) return;
        for (int p = p0; p < p1; ++p) {
            const Eight<T> piece = Eight<T>::of(row.row + row.head + (int64_t)p * N, true);
            bool done = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                done = done || f(piece.at(i), row.head + p * N + i);
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
            if (done) return;
        }
        if (has_tail)
            for (int v = row.head + row.full * N; v < row.vocab; ++v) if (f(to_f32(row.row[v]), v)) return;
    };
    u64 sum = 0;
    int equal_here = 0;
    walk([&](float x, int) __attribute__((always_inline)) {
        sum += weight(x > least ? x : -INFINITY);
        equal_here += x == least;
        return false;
    });
    u64 all;
    if (equal) base_ties += sum_before(s, (u64)equal_here, all);
    sum += ties_left(base_ties, equal_here) * w_least;
    base += sum_before(s, sum, all);
    if (sum && !((double)base > target && base) && ((double)(base + sum) > target || base + sum == total)) {
        int chosen = 0;
        float logit = m;
        walk([&](float x, int v) {
            if (!(x > least) && !(x == least && base_ties++ < equal)) return false;
            const u64 wx = weight(x);
            if (!wx) return false;
            chosen = v; logit = x;
            base += wx;
            return (double)base > target;
        });
        write(chosen, logit, total);
    }
}
};

template <int LANES, typename T>
__global__ void __launch_bounds__(LANES, 4) k_sample(const SampleArgs a) { Sampling<LANES>::template run<T>(a); }

template <int LANES>
void launch_sample(const SampleArgs &a, int dtype, int rows, hipStream_t s)
{
    if (dtype == EL_F32) hipLaunchKernelGGL((k_sample<LANES, float>), dim3(rows), dim3(LANES), 0, s, a);
    else if (dtype == EL_F16) hipLaunchKernelGGL((k_sample<LANES, f16_t>), dim3(rows), dim3(LANES), 0, s, a);
    else hipLaunchKernelGGL((k_sample<LANES, bf16_t>), dim3(rows), dim3(LANES), 0, s, a);
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
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    for (int32_t first = 0; first < rows; first += kRowsOfLaunch) {
        const int32_t n = rows - first < kRowsOfLaunch ? rows - first : kRowsOfLaunch;
        auto from = [&](auto *p) { return p ? p + first : nullptr; };
        const el_attn_sample_rule here{rule->temperature, rule->top_k, rule->top_p, rule->min_p,
                                       from(rule->row_temperature), from(rule->row_top_k), from(rule->row_top_p), from(rule->row_min_p)};
        const SampleArgs a{(const char *)logits + first * (row_stride * es), row_stride * es, vocab, uniform + first, here, tokens + first, from(logprob), kPowers, n,
                           n > kComputeUnits && n <= kOrdered && (rule->row_top_k || rule->row_top_p)};
        if (n > kComputeUnits) launch_sample<512>(a, dtype, n, s);
        else launch_sample<1024>(a, dtype, n, s);
    }
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}
