// What a row of logits says about the next token: log-probability of a given one, entropy, the best alternatives.
//
//   log p(x) = (x - m) - log S,  S = sum exp(x - m),  entropy = log S - W / S,  W = sum exp(x - m) (x - m)
//
// with m the largest logit: the differences are exact to a rounding whatever m is, a row of the type's lowest value included.
//
// Bound by HBM where rows are many: every logit is read once.  A workgroup holds a chunk of a row in registers, so maximum, sums
// and alternatives are passes over registers.  Rows start anywhere (an odd vocabulary): chunks are cut at 16-byte boundaries of
// memory, and the elements at a row's ends that do not fill 16 bytes are a lane's each.
// Alternatives: the k-th largest of the 256 lanes' maxima has k elements at or above it, so whatever lies below it is none of the
// chunk's k best; about as many as k are left, and are ranked by counting.  k_score_join joins the chunks of a row.
#include <cfloat>
#include <cmath>
#include "mfma.h"

namespace el {
namespace {

constexpr int kMaxAlternatives = 64;
constexpr int kLanes = 256;
constexpr int kCandidates = 1024;        // of a chunk that are ranked by counting
constexpr int kFillWorkgroups = 512;     // chunks get smaller until about so many workgroups share the logits: two a compute unit
constexpr int kRowLanes = 1024, kRowsWhole = 256;
constexpr int32_t kMaxVocab = 1 << 19;
constexpr int kListMax = 2048;           // entries of a row's lists, which k_score_join holds in registers: 32 chunks of the largest vocabulary in fp32
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef unsigned long long Key;

struct ScoreArgs {
    const char *logits;
    int64_t row_stride;                  // bytes
    int vocab, k, chunks, pieces;        // pieces of 16 bytes of a chunk
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_index;
    f4 *stats;                           // [row][chunk] m, S, W
    Key *keys;                           // [row][chunk][k] descending; 0: none
};

// What orders alternatives: the value, then the lower index.
__device__ __forceinline__ unsigned order32(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);                     // (-0 counts as 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }
__device__ __forceinline__ Key key_of(float x, int v) { return ((Key)order32(x) << 32) | (0xffffffffu - (unsigned)v); }

template <typename T> struct Piece;      // 16 bytes of logits
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ u4 none() { return u4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }      // all -inf
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float at(u4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
    static __device__ __forceinline__ u4 none() { return u4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
};
template <> struct Piece<f16_t> {
    static constexpr int N = 8;
    // (a bit cast of a vector's element itself takes element 0 whatever the index: through a copy)
    static __device__ __forceinline__ float at(u4 v, int i) { const unsigned u = v[i >> 1]; return (float)__builtin_bit_cast(h2, u)[i & 1]; }
    static __device__ __forceinline__ u4 none() { return u4{0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u}; }
};

// How many of the first n keys of a list that goes on with at least 7 zeros are larger: 8 in flight at a time.
__device__ __forceinline__ int rank_in(const Key *list, int n, Key key)
{
    int rank = 0;
    for (int o = 0; o < n; o += 8) {
        Key other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = list[o + i];
#pragma unroll
        for (int i = 0; i < 8; ++i) rank += other[i] > key;
    }
    return rank;
}

struct Sums { float m, S, W; };
__device__ __forceinline__ Sums join(Sums a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    // (nothing above -inf on a side: its sums are 0, or NaN, and stay; a difference beyond the type's range is one whose power is 0)
    const float da = a.m == -INFINITY ? 0.f : fmaxf(a.m - m, -1e30f), db = b.m == -INFINITY ? 0.f : fmaxf(b.m - m, -1e30f);
    const float fa = __builtin_amdgcn_exp2f(da * kLog2e), fb = __builtin_amdgcn_exp2f(db * kLog2e);
    return Sums{m, fa * a.S + fb * b.S, fa * (a.W + da * a.S) + fb * (b.W + db * b.S)};
}

__device__ __forceinline__ float first_lane(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
__device__ __forceinline__ float log_of(float S) { return __builtin_amdgcn_logf(S) * kLn2; }

// The given token's logit; where there is none, NaN (beyond the vocabulary) or +inf (no token given).
template <typename T>
__device__ __forceinline__ float given_logit(const ScoreArgs &a, int64_t r)
{
    if (!a.logprob) return 0.f;
    const int t = a.tokens[r];
    if (t < 0 || t >= a.vocab) return t < 0 ? INFINITY : NAN;
    const float x = to_f32(((const T *)(a.logits + r * a.row_stride))[t]);
    return x == INFINITY ? NAN : x;                                  // (a logit of +inf has no log-probability)
}
// logprob and entropy of a row, by one lane.
__device__ __forceinline__ void write_row(const ScoreArgs &a, int64_t r, Sums s, float given)
{
    const bool none = s.S == 0.f;                                    // no token may follow: `given` is -inf, or NaN
    if (a.entropy) a.entropy[r] = none ? 0.f : log_of(s.S) - s.W / s.S;
    if (a.logprob) a.logprob[r] = given == INFINITY ? 0.f : none ? given : (given - s.m) - log_of(s.S);
}
__device__ __forceinline__ void write_alternative(const ScoreArgs &a, int64_t r, int i, Key key, float m, float log_S)
{
    a.top_logprob[r * a.k + i] = key ? (value_of((unsigned)(key >> 32)) - m) - log_S : -INFINITY;
    a.top_index[r * a.k + i] = key ? (int)(0xffffffffu - (unsigned)key) : -1;
}

// Where a row's `full` pieces of 16 bytes lie: the first behind `head` elements, at a 16-byte boundary.
struct Row { const char *row; int head, full; };
template <typename T>
__device__ __forceinline__ Row row_at(const ScoreArgs &a, int64_t r)
{
    const char *const row = a.logits + r * a.row_stride;
    const int head = min((int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T), a.vocab);
    return Row{row, head, (a.vocab - head) / Piece<T>::N};
}
// Piece p, if it is below `end`; -inf otherwise.
template <typename T>
__device__ __forceinline__ u4 load_piece(const Row &x, int p, int end)
{
    if (p < end) return __builtin_nontemporal_load((const u4 *)(x.row + x.head * (int)sizeof(T)) + p);
    return Piece<T>::none();
}
// The elements around the pieces, fewer than 2 N, are one lane's each: index of lane t's, or -1.
template <typename T>
__device__ __forceinline__ int edge_of(const Row &x, int t, int vocab)
{
    const int i = t < x.head ? t : t + x.full * Piece<T>::N;
    return t < 2 * Piece<T>::N && i < vocab ? i : -1;
}

template <typename T>
__device__ __forceinline__ float largest(u4 v)
{
    float m = Piece<T>::at(v, 0);
#pragma unroll
    for (int i = 1; i < Piece<T>::N; ++i) m = fmaxf(m, Piece<T>::at(v, i));
    return m;
}
__device__ __forceinline__ void add_term(float x, float ref, float &S, float &W)
{
    const float d = x - ref, e = __builtin_amdgcn_exp2f(d * kLog2e);
    S += e;
    W = fmaf(e, fmaxf(d, -1e4f), W);                                 // (a banned token: 0, not 0 * inf)
}

// The k-th largest of the numbers of `COUNT` x 64 lanes, without its bits below LOW (0: fewer than k are above 0).
template <int LOW, int COUNT>
__device__ __forceinline__ unsigned kth_of(const unsigned (&mine)[COUNT], int k)
{
    unsigned bound = 0;
#pragma unroll
    for (int bit = 31; bit >= LOW; --bit) {
        const unsigned t = bound | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) n += __popcll(__ballot(mine[i] >= t));
        if (n >= k) bound = t;
    }
    return bound;
}

// A chunk of up to NV pieces a lane of one row; LANES 1024: the whole row.  Grid: rows x chunks.
// With 1024 lanes a compute unit holds two rows where NV is at most 8 (64 registers; left alone the compiler takes 70), so that one is loaded while the
// other is computed: 512 rows of 65000 in bf16, 8 alternatives, 19.9 us, 24.6 with one; 1024 of 50265 32.2 / 44.2; 300 of 30000 in fp32 14.2 / 17.1.
template <typename T, int NV, int LANES>
__global__ void __launch_bounds__(LANES, LANES == kRowLanes && NV <= 8 ? 8 : 1) k_score_chunk(const ScoreArgs a)
{
    constexpr int N = Piece<T>::N, WAVES = LANES / 64;
    __shared__ unsigned best[256];
    __shared__ __attribute__((aligned(16))) Key cand[kCandidates + 8];
    __shared__ Sums part[WAVES];
    __shared__ int count;
    __shared__ Key top[WAVES];
    __shared__ int equal[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t r = blockIdx.x / a.chunks;
    const int chunk = blockIdx.x - (int)r * a.chunks;
    const Row row = row_at<T>(a, r);
    const int used = NV < 16 ? NV : (a.pieces + LANES - 1) / LANES;          // (uniform) pieces that some lane has
    const int from = chunk * a.pieces + tid, end = min((chunk + 1) * a.pieces, row.full);           // this lane's pieces: LANES apart
    if (tid == 0) count = 0;
    if (a.k)
        for (int i = tid; i < kCandidates + 8; i += LANES) cand[i] = 0;

    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        v[j] = Piece<T>::none();
        if (j < used) v[j] = load_piece<T>(row, from + j * LANES, end);
    }
    const int edge = chunk == 0 ? edge_of<T>(row, tid, a.vocab) : -1;
    const float x_edge = edge >= 0 ? to_f32(((const T *)row.row)[edge]) : -INFINITY;
    const float given = a.chunks == 1 && tid == 0 ? given_logit<T>(a, r) : 0.f;
    float most[NV], m = x_edge;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        most[j] = -INFINITY;
        if (j >= used) continue;
        most[j] = largest<T>(v[j]);
        m = fmaxf(m, most[j]);
        asm volatile("" : "+v"(v[j]));                               // (one piece unpacked at a time)
    }
    if constexpr (LANES == 256) {
        best[tid] = m > -INFINITY ? order32(m) : 0u;
    } else {                                                         // (of four lanes each: 256 numbers again)
        float m4 = fmaxf(m, quad_xor1(m));
        m4 = fmaxf(m4, quad_xor2(m4));
        if (tid % 4 == 0) best[tid / 4] = m4 > -INFINITY ? order32(m4) : 0u;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float ref = m == -INFINITY ? 0.f : m;
    float S = 0.f, W = 0.f;
    add_term(x_edge, ref, S, W);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j >= used) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) add_term(Piece<T>::at(v[j], i), ref, S, W);
        asm volatile("" : "+v"(v[j]));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { S += __shfl_xor(S, o, 64); W += __shfl_xor(W, o, 64); }
    if (lane == 0) part[w] = Sums{m, S, W};
    __syncthreads();
    const bool whole = a.chunks == 1;
    Sums s = part[lane % WAVES];
#pragma unroll
    for (int o = WAVES / 2; o > 0; o >>= 1) s = join(s, Sums{__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.W, o, 64)});
    // (lanes join the same numbers in another order: lane 0's result for all, to the bit)
    s = Sums{first_lane(s.m), first_lane(s.S), first_lane(s.W)};
    if (tid == 0) {
        if (whole) write_row(a, r, s, given);
        else a.stats[blockIdx.x] = f4{s.m, s.S, s.W, 0.f};
    }
    if (a.k == 0) return;
    const float log_S = log_of(s.S);
    auto emit = [&](int i, Key key) __attribute__((always_inline)) {
        if (whole) write_alternative(a, r, i, key, s.m, log_S);
        else a.keys[(int64_t)blockIdx.x * a.k + i] = key;
    };
    const unsigned maxima[4] = {best[lane], best[lane + 64], best[lane + 128], best[lane + 192]};
    const unsigned bound = kth_of<16>(maxima, a.k);
    const float least = bound ? value_of(bound) : -FLT_MAX;
    auto collect = [&](float x, int index) __attribute__((always_inline)) {
        if (x >= least) {
            const int at = atomicAdd(&count, 1);
            if (at < kCandidates) cand[at] = key_of(x, index);
        }
    };
    collect(x_edge, edge);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (!__ballot(most[j] >= least)) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) collect(Piece<T>::at(v[j], i), row.head + (from + j * LANES) * N + i);
    }
    __syncthreads();
    int n = count;
    if (n > kCandidates && bound) {
        // Ties, mostly: what is larger than the exact bound, and of what equals it, looked through in order of index, the first that still
        // lack.  (Pieces are read again: rare, and registers are short.)  1024 rows of 128003 zeros in fp32, 20 alternatives, 257 us, one at a
        // time 2260.
        const float exact = value_of(kth_of<0>(maxima, a.k));
        __syncthreads();
        if (tid == 0) count = 0;
        for (int i = tid; i < kCandidates + 8; i += LANES) cand[i] = 0;
        __syncthreads();
        auto above = [&](float x, int index) __attribute__((always_inline)) {
            if (x > exact) {
                const int at = atomicAdd(&count, 1);
                if (at < kCandidates) cand[at] = key_of(x, index);
            }
        };
        above(x_edge, edge);
#pragma unroll 1
        for (int j = 0; j < used; ++j) {
            const u4 again = load_piece<T>(row, from + j * LANES, end);
#pragma unroll
            for (int e = 0; e < N; ++e) above(Piece<T>::at(again, e), row.head + (from + j * LANES) * N + e);
        }
        __syncthreads();
        n = count;
        // the elements before the pieces, the pieces, those behind: a lane's lie behind those of the lanes before it
#pragma unroll 1
        for (int j = -1; j <= used && n < a.k; ++j) {
            unsigned flags = 0;
            int index = edge;
            if (j < 0 || j == used) {
                flags = edge >= 0 && (edge < row.head) == (j < 0) && x_edge == exact;
            } else {
                const u4 again = load_piece<T>(row, from + j * LANES, end);
                index = row.head + (from + j * LANES) * N;
#pragma unroll
                for (int e = 0; e < N; ++e) flags |= (unsigned)(Piece<T>::at(again, e) == exact) << e;
            }
            int upto = __popc(flags);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int other = __shfl_up(upto, o, 64);
                if (lane >= o) upto += other;
            }
            if (lane == 63) equal[w] = upto;
            __syncthreads();
            int at = n + upto - __popc(flags);
            for (int i = 0; i < WAVES; ++i) {
                if (i < w) at += equal[i];
                n += equal[i];
            }
            for (; flags && at < a.k; flags &= flags - 1) cand[at++] = key_of(exact, index + __ffs((int)flags) - 1);
            __syncthreads();
        }
        if (count < a.k) n = min(n, a.k);
    }
    if (n <= kCandidates) {
        for (int c = tid; c < n; c += LANES) {
            const Key key = cand[c];
            const int rank = rank_in(cand, n, key);
            if (rank < a.k) emit(rank, key);
        }
        for (int c = n + tid; c < a.k; c += LANES) emit(c, 0);
        return;
    }
    Key last = ~(Key)0;
    for (int i = 0; i < a.k; ++i) {
        Key mine = 0;
        auto better = [&](float x, int index) __attribute__((always_inline)) {
            const Key key = x >= least ? key_of(x, index) : 0;
            if (key < last && key > mine) mine = key;
        };
        better(x_edge, edge);
#pragma unroll 1
        for (int j = 0; j < NV; ++j) {                               // (read again: rare, and registers are short)
            const u4 again = load_piece<T>(row, from + j * LANES, end);
#pragma unroll
            for (int e = 0; e < N; ++e) better(Piece<T>::at(again, e), row.head + (from + j * LANES) * N + e);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const Key other = __shfl_xor(mine, o, 64);
            mine = mine > other ? mine : other;
        }
        __syncthreads();
        if (lane == 0) top[w] = mine;
        __syncthreads();
        last = 0;
#pragma unroll 4
        for (int j = 0; j < WAVES; ++j) last = top[j] > last ? top[j] : last;
        if (tid == 0) emit(i, last);
    }
}

// The chunks of a row joined: one row a workgroup.  The lists are descending; taken across, first entries first, they are numbers of 256 lanes
// whose k-th largest maximum bounds the k best as in a chunk.  Bound by latency: everything is requested at once.
template <typename T>
__global__ void __launch_bounds__(kLanes) k_score_join(const ScoreArgs a)
{
    extern __shared__ __attribute__((aligned(16))) Key list[];       // [chunks * k + 8] what is left, and zeros
    __shared__ Sums part[4];
    __shared__ unsigned best[kLanes];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t r = blockIdx.x;
    const int total = a.chunks * a.k;
    const Key *const keys = a.keys + r * total;
    auto key_at = [&](int t) __attribute__((always_inline)) {        // entry t / chunks of list t % chunks
        const int i = t / a.chunks;
        return t < total ? keys[(t - i * a.chunks) * a.k + i] : 0;
    };
    constexpr int HELD = kListMax / kLanes;
    Key key[HELD], most = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j) key[j] = key_at(tid + j * kLanes);
    const float given = tid == 0 ? given_logit<T>(a, r) : 0.f;
    Sums s{-INFINITY, 0.f, 0.f};
    for (int c = tid; c < a.chunks; c += kLanes) {
        const f4 v = a.stats[r * a.chunks + c];
        s = join(s, Sums{v[0], v[1], v[2]});
    }
    if (tid == 0) count = 0;
    for (int i = tid; i < total + 8; i += kLanes) list[i] = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j) most = key[j] > most ? key[j] : most;
    best[tid] = (unsigned)(most >> 32);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s = join(s, Sums{__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.W, o, 64)});
    if (lane == 0) part[w] = s;
    __syncthreads();
    s = join(join(part[0], part[1]), join(part[2], part[3]));
    if (tid == 0) write_row(a, r, s, given);
    if (a.k == 0) return;
    const unsigned maxima[4] = {best[lane], best[lane + 64], best[lane + 128], best[lane + 192]};
    // (0: no alternative.  64 entries are ranked sooner than bounded: 2000 rows of 50265 in bf16, 8 alternatives, 51.7 us, 53.2 bounded)
    const Key least = total <= 64 ? (Key)1 : max((Key)kth_of<16>(maxima, a.k) << 32, (Key)1);
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (key[j] >= least) list[atomicAdd(&count, 1)] = key[j];
    __syncthreads();
    const int n = count;
    const float log_S = log_of(s.S);
    for (int c = tid; c < n; c += kLanes) {
        const Key k = list[c];
        const int rank = rank_in(list, n, k);
        if (rank < a.k) write_alternative(a, r, rank, k, s.m, log_S);
    }
    for (int i = n + tid; i < a.k; i += kLanes) write_alternative(a, r, i, 0, s.m, log_S);
}

// How a call is cut: pieces a lane, chunks of a row.
static_assert(kMaxVocab / 4 / (16 * kLanes) * kMaxAlternatives <= kListMax, "the fewest chunks of a row");
struct ScorePlan { int form, lanes, chunks, pieces; size_t stats_bytes, workspace; };

ScorePlan plan_score(int element_size, int32_t rows, int32_t vocab, int32_t k)
{
    const int n = 16 / element_size;
    const int pieces = vocab < n ? 1 : vocab / n;                    // full ones of a row, at most
    ScorePlan p;
    p.lanes = kLanes;
    p.form = 16;
    auto chunks = [&](int form) { return (pieces + form * kLanes - 1) / (form * kLanes); };
    // The more a workgroup holds, the fewer lists there are to join: 1024 rows of 128003 in fp32, 20 alternatives, 111 us with 8 pieces a
    // lane, 96 with 16, which take two rounds of workgroups.
    // A row that one workgroup holds is not cut, unless rows are few and it has more than 8 pieces a lane: 300 rows of 8000 in bf16, 8 alternatives,
    // 6.6 us, 10.2 cut; of 32001 12.4 / 14.0; 64 rows of 32001 9.5, 8.0 as below.
    const int alone = rows > kRowsWhole ? 16 : 8;
    while (p.form > 1 && (chunks(p.form) > 1 || p.form > alone) && (int64_t)rows * chunks(p.form) < (p.form > 8 ? 2 * kFillWorkgroups : kFillWorkgroups) && chunks(p.form / 2) * k <= kListMax) p.form /= 2;
    p.chunks = chunks(p.form);
    while (p.form > 1 && chunks(p.form / 2) == p.chunks) p.form /= 2;
    // Rows that 1024 lanes hold: one launch, a row a workgroup.  256 rows of 50265 in bf16, 8 alternatives, 13.1 us, 16.1 cut; 512 18.9 / 21.7;
    // 1024 32.2 / 32.4, of 33000 29.5 / 27.3, of 20000 in fp32 23.0 / 24.9; 300 of 128003, whose registers leave room for one such workgroup a compute
    // unit, 35 / 27.
    if (p.chunks > 1 && rows <= (pieces <= 8 * kRowLanes ? 4 * kRowsWhole : kRowsWhole) && pieces <= 16 * kRowLanes) {
        p.lanes = kRowLanes; p.chunks = 1;
        p.form = pieces <= 4 * kRowLanes ? 4 : pieces <= 8 * kRowLanes ? 8 : 16;
    }
    p.pieces = (pieces + p.chunks - 1) / p.chunks;                   // chunks of one size
    p.stats_bytes = p.workspace = 0;
    if (p.chunks > 1) {
        p.stats_bytes = align_up((size_t)rows * p.chunks * sizeof(f4), 256);
        p.workspace = p.stats_bytes + (size_t)rows * p.chunks * k * sizeof(Key);
    }
    return p;
}

template <typename T>
void launch_score(const ScoreArgs &a, const ScorePlan &p, int rows, hipStream_t s)
{
    const dim3 grid((unsigned)(rows * p.chunks)), block(kLanes);
    if (p.lanes == kRowLanes) {
        if (p.form == 16) hipLaunchKernelGGL((k_score_chunk<T, 16, kRowLanes>), grid, dim3(kRowLanes), 0, s, a);
        else if (p.form == 8) hipLaunchKernelGGL((k_score_chunk<T, 8, kRowLanes>), grid, dim3(kRowLanes), 0, s, a);
        else hipLaunchKernelGGL((k_score_chunk<T, 4, kRowLanes>), grid, dim3(kRowLanes), 0, s, a);
    } else if (p.form == 16) hipLaunchKernelGGL((k_score_chunk<T, 16, kLanes>), grid, block, 0, s, a);
    else if (p.form == 8) hipLaunchKernelGGL((k_score_chunk<T, 8, kLanes>), grid, block, 0, s, a);
    else if (p.form == 4) hipLaunchKernelGGL((k_score_chunk<T, 4, kLanes>), grid, block, 0, s, a);
    else if (p.form == 2) hipLaunchKernelGGL((k_score_chunk<T, 2, kLanes>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_score_chunk<T, 1, kLanes>), grid, block, 0, s, a);
    if (p.chunks > 1) hipLaunchKernelGGL((k_score_join<T>), dim3(rows), block, ((size_t)p.chunks * a.k + 8) * sizeof(Key), s, a);
}

constexpr int64_t kMaxChunks = (int64_t)1 << 23;                     // rows x chunks: a launch has fewer than 2^32 threads

bool valid_sizes(int32_t rows, int32_t vocab, int32_t k)
{
    return rows >= 1 && vocab >= 1 && k >= 0 && k <= kMaxAlternatives && rows <= kMaxChunks;
}

} // namespace
} // namespace el

extern "C" int32_t el_attn_max_alternatives(void) { return el::kMaxAlternatives; }

extern "C" size_t el_attn_score_workspace_bytes(int32_t rows, int32_t vocab, int32_t k)
{
    using namespace el;
    if (!valid_sizes(rows, vocab, k) || vocab > kMaxVocab) return 0;
    const size_t two = plan_score(2, rows, vocab, k).workspace, four = plan_score(4, rows, vocab, k).workspace;
    return two > four ? two : four;
}

extern "C" el_status el_attn_score_tokens(el_dtype dtype, const void *logits, int64_t row_stride, int32_t rows, int32_t vocab,
                                          const int32_t *tokens, float *logprob, float *entropy,
                                          int32_t k, float *top_logprob, int32_t *top_index,
                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (dtype != EL_F32 && dtype != EL_F16 && dtype != EL_BF16) return EL_ERR_UNSUPPORTED;
    if (!logits || !valid_sizes(rows, vocab, k)) return EL_ERR_INVALID_ARG;
    if (vocab > kMaxVocab) return EL_ERR_UNSUPPORTED;
    if ((logprob && !tokens) || (k > 0 && (!top_logprob || !top_index))) return EL_ERR_INVALID_ARG;
    if ((rows > 1 && row_stride < vocab) || row_stride > ((int64_t)1 << 44)) return EL_ERR_INVALID_ARG;
    const int64_t es = (int64_t)dtype_size(dtype);
    if ((uintptr_t)logits % (size_t)es != 0 || out_of_reach(rows, row_stride * es)) return EL_ERR_INVALID_ARG;
    if (((uintptr_t)tokens | (uintptr_t)logprob | (uintptr_t)entropy | (uintptr_t)top_logprob | (uintptr_t)top_index) & 3) return EL_ERR_INVALID_ARG;
    const ScorePlan p = plan_score((int)es, rows, vocab, k);
    if ((int64_t)rows * p.chunks > kMaxChunks) return EL_ERR_INVALID_ARG;
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return EL_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 15) return EL_ERR_INVALID_ARG;
    }
    const ScoreArgs a{(const char *)logits, row_stride * es, vocab, k, p.chunks, p.pieces, tokens, logprob, entropy, top_logprob, top_index,
                      (f4 *)workspace, (Key *)((char *)workspace + p.stats_bytes)};
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    if (dtype == EL_F32) launch_score<float>(a, p, rows, s);
    else if (dtype == EL_F16) launch_score<f16_t>(a, p, rows, s);
    else launch_score<bf16_t>(a, p, rows, s);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}
