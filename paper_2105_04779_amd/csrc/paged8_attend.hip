// Attention of one new token per query row over pages of 8-bit codes with a scale for each block of positions and head.
//
//   s_t = scale ks_t (q.k_t) (capped, biased by distance),  out = sum_t softmax(s)_t vs_t v_t,  lse = log sum_t exp s_t
//
// with codes k_t, v_t and scales ks_t, vs_t, over the positions that are there: below the length, inside the window, in a page of the pool.
//
// Bound by HBM where sequences are many or long: a byte of a key or value is read once and used by the query rows that share the key head.  At half the
// bytes of 16-bit storage the vector ALU has half the time for a position, so codes go the shortest way into the matrix unit:
//   - A wavefront works alone on tiles of 32 positions, codes straight from memory in registers, the next tile under way while one is
//     computed; no LDS.  Codes of both formats are 16-bit numbers exactly (two values an instruction for e4m3).
//   - A request covers whole lines: 8 lanes read 128 bytes of a key, which are past the caches then; two rows' lanes trade halves (DPP) to get the operands' order.
//     With 16 rows of 64 bytes a request, two requests a line, the stream stayed at 4.7 TB/s without any arithmetic, however many wavefronts, and 5.3 with whole ones.
//   - The compiler waits for requests by count, by the shortest way through the loop: all ways have as many.  Positions that are not there are replaced by others,
//     page numbers come through the scalar cache a tile ahead, the last tile is a copy of the loop's body.
//   - S^T = K Q^T: rows of K are positions, a lane's 16 bytes of a row are two operands (the inner index may be in any order, and Q's is in the same).
//     Row m of product x is position 8 (m / 4) + 4 x + m % 4, so a lane of S^T holds 8 positions that are neighbours: they are the 8 inner indices that it
//     supplies to O^T += V^T P^T, P never leaves the registers, and the lane's 8 rows of V lie one behind the other in a page.
//   - V^T's operand needs 8 positions of a column in a lane: a lane loads d / 16 bytes of each of its 8 rows and pairs the bytes of two rows (v_perm)
//     before they are converted.
//   - ks multiplies a score in the subtraction of the running maximum, vs multiplies p before that is split into bf16 parts, which have fp32's range.
// us with the join, twelve passes a captured graph, inputs in no cache: 64 sequences of 1024 to 4096 positions, 32 heads on 8 key heads of 128, e4m3, 337 MB, 79 (4.2 TB/s);
// two of 100000 to 131072 in int8, 473 MB, 101 (4.7); 16 of up to 8192, 8 key heads of 256, 337 MB, 72 to 75.  64 columns, half a line a request: 16 heads, 64 of 1024 to 4096, 337 MB,
// 105 (3.2 TB/s); two of 100000 to 131072, 474 MB, 138 (3.4); 512 continuations of up to 256, 152 MB, 55 to 57; one sequence of 613, 11.9.  (Three passes a graph, which
// leaves some 6 more on each: the first 112 with half lines and waits for all that was under way, 91 with twelve wavefronts a compute unit, 86; the second 143, 118.)
// Of the first in other forms: fp32 queries 85; cap, window and slopes 87; a scale for every position or pages of 10 (not FAST) 103 and 104.  32 rows on each of 8 key heads, 32 of
// 1024 to 4096, 168 MB, 68; 40 rows, which read and convert the codes twice, 102; 32 rows at 256 columns 142.
// Work: paged_spans.h.
#include <type_traits>
#include "paged8.h"
#include "paged_spans.h"

namespace el {
namespace {

constexpr int TP = 32;                   // positions of a tile
constexpr int kRor8 = 0x128;             // 16 lanes rotated by 8

struct Attend8Args : AttendArgs {
    ScaleView s;
    int dtype;                           // of the queries
    int step_slots, step_rest;           // pages and positions that 32 positions are
};

// Form of a wavefront: format, d_head padded, query rows in groups of 16, the queries' type (EL_F32: three bf16 parts, which hold any type's bits).
// FAST: pages and blocks are multiples of 8 positions, so a lane's 8 positions have one page and one scale.
// A probability times its scale is three bf16 parts, which hold its 24 bits, whatever the result's type.  Two (16 bits) would round one result in a thousand
// to bf16 the other way, fourteen to fp16, and save little, us with two / three: 64 sequences of 1024 to 4096 on 8 key heads of 128 80.4 / 79.4, 512 of up to 256, 16 heads of 64,
// 54.0 / 56.2, 32 of 1024 to 4096, 32 rows on each of 8 key heads of 128, 65.5 / 67.9, 16 of up to 8192 at 256 columns 70.7 / 72.2, one of 613 11.4 / 11.7.
template <int FMT_, int DP_, int RG_, int QT_, bool FAST_> struct Form8 {
    static constexpr int FMT = FMT_, DP = DP_, RG = RG_, QT = QT_, NP = 3, QP = QT == EL_F32 ? 3 : 1;
    static constexpr bool FAST = FAST_;
    static constexpr int LDS = RG * DP * 64 + 256;                   // of a wavefront that shares its sequence: results, (m, l)
    // wavefronts that a compute unit holds, by registers (twelve of 128 columns would fit, and take 6 % longer: 64 sequences of 1024 to 4096 on 8 key heads)
    static constexpr int PER_CU = DP == 256 || (DP == 128 && RG * QP == 6) ? 4 : DP == 128 || RG * QP > 2 ? 8 : RG == 2 ? 12 : 16;
    static constexpr int ROOM = 163840 / LDS, WAVES = ROOM >= 8 && PER_CU >= 8 ? 8 : 4;
};

template <int N> struct Bytes;
template <> struct Bytes<4> { typedef unsigned T; static __device__ __forceinline__ unsigned at(T v, int) { return v; } };
template <> struct Bytes<8> { typedef u2 T; static __device__ __forceinline__ unsigned at(T v, int i) { return v[i]; } };
template <> struct Bytes<16> { typedef u4 T; static __device__ __forceinline__ unsigned at(T v, int i) { return v[i]; } };

// Codes as 16-bit numbers, exactly: bytes (0, 1) or (2, 3) of a dword; byte I of two dwords.
template <int FMT, bool BF16> struct Number;
template <bool BF16> struct Number<EL_E4M3, BF16> {
    template <bool HIGH> static __device__ __forceinline__ unsigned two(unsigned w)
    {
        if constexpr (BF16) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HIGH));
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, HIGH));
    }
    // (the two bytes' neighbours are paired by the same instruction, and used by I ^ 1)
    template <int I> static __device__ __forceinline__ unsigned of_two(unsigned a, unsigned b) { return two<(I & 1) != 0>(__builtin_amdgcn_perm(b, a, I & 2 ? 0x07030602u : 0x05010400u)); }
};
template <bool BF16> struct Number<EL_INT8, BF16> {
    template <int I> static __device__ __forceinline__ float at(unsigned w) { return (float)(int)__builtin_amdgcn_sbfe(w, 8 * I, 8); }
    static __device__ __forceinline__ unsigned pair(float x, float y)
    {
        if constexpr (BF16) return __builtin_bit_cast(unsigned, __builtin_convertvector(f2{x, y}, b2));
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(x, y));
    }
    template <bool HIGH> static __device__ __forceinline__ unsigned two(unsigned w) { return pair(at<HIGH ? 2 : 0>(w), at<HIGH ? 3 : 1>(w)); }
    template <int I> static __device__ __forceinline__ unsigned of_two(unsigned a, unsigned b) { return pair(at<I>(a), at<I>(b)); }
};

template <class F>
__global__ void __launch_bounds__(64 * F::WAVES, F::PER_CU / 4) k_coded_attend(const Attend8Args a)
{
    constexpr int DP = F::DP, RG = F::RG, QP = F::QP, NP = F::NP, DT16 = DP / 16, KC = DP / 64, ITEMS = DP / 16, SC = F::FAST ? 1 : 8;
    constexpr bool FAST = F::FAST;
    constexpr bool BF16 = F::QT != EL_F16;
    typedef Number<F::FMT, BF16> KN;
    typedef Number<F::FMT, true> VN;
    typedef Bytes<DP / 16> VB;
    typedef typename VB::T VT;
    extern __shared__ __attribute__((aligned(16))) char shared[];   // (workgroups of several wavefronts) [wavefront] results, (m, l)

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = a.kv_heads * a.row_blocks;
    int span = blockIdx.x / units, unit = blockIdx.x - span * units;
    if (a.near && (span / kDies + 1) * kDies * units <= (int)gridDim.x) {            // workgroups go round the dies: a die takes a span's units
        const int first = span / kDies * kDies, i = blockIdx.x - first * units;
        span = first + i % kDies;
        unit = i / kDies;
    }
    const int kvh = unit % a.kv_heads, row0 = unit / a.kv_heads * a.rows;
    const int64_t scale_page = (int64_t)a.kv_heads * a.s.per;

    Start st{span, 0, 0, 0, 1, false};
    if (a.spans && !find_span(a, span, TP, st)) return;
    // the pieces of this span: the tiles of one sequence after the other
    for (;;) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));          // (what follows from it is worked out anew for a piece, instead of being held over all of them)
    const int r16 = lane & 15, g = lane >> 4;
    const int64_t b = st.b;
    const int len = length_of(a, st.b), first = a.window ? max(0, len - a.window) : 0;
    const int2 range = tile_range(a, len, TP);
    const int tiles = range.y - range.x;
    if (a.spans && tiles == 0) { ++st.b; continue; }                 // (there is a tile to come: st.b stays below B)
    int t0 = range.x, nt = tiles, pieces = 1;
    if (a.spans) {
        t0 += st.at - st.before;
        nt = min(range.y - t0, st.end - st.at);
        pieces = (st.before + tiles - 1) / st.T - st.before / st.T + 1;       // (aligned: st.before is a multiple of T)
        if (t0 == range.x && unit == 0 && lane == 0) a.pieces[b] = int2{span + st.b, pieces};
    } else {                                                         // the workgroup's wavefronts share the sequence
        const int each = (tiles + a.waves - 1) / a.waves, skip = min(wave * each, tiles);
        t0 += skip;
        nt = min(each, tiles - skip);
    }

    // ---- the way of the tiles ----
    // A lane's chunk c of 16 bytes in a row of K, and its place in a row of V; columns beyond d_head are some of those below it: in K zeros of the
    // queries meet them, in V their results are nobody's.  Request (x, n) reads whole lines of 8 rows of K; the lanes trade half of them (scores).
    constexpr bool LINES = DP >= 128;
    auto k_col = [&](int c) __attribute__((always_inline)) { return LINES ? 128 * (c >> 1) + 32 * g + 16 * (c & 1) : 64 * c + 16 * g; };
    const int v_col = min(r16 * (DP / 16), a.d - DP / 16), v_row = 8 * g;
    constexpr int KR = LINES ? 2 : 1;       // requests for the rows of a product
    auto k_row = [&](int n) __attribute__((always_inline)) { return LINES ? 16 * n + 8 * (r16 >> 2 & 1) + (r16 & 3) : 8 * (r16 >> 2) + (r16 & 3); };
    const char *const Kh = a.c.K + kvh * a.c.head, *const Vh = a.c.V + kvh * a.c.head + v_col;
    const float *const Ks = a.s.K + (int64_t)kvh * a.s.per, *const Vs = a.s.V + (int64_t)kvh * a.s.per;
    const int32_t *const table = a.c.table + b * a.c.table_stride;
    const unsigned page_size = (unsigned)a.c.page_size, last_slot = len > 0 ? (unsigned)(len - 1) / page_size : 0;
    auto in_pool = [&](int page) __attribute__((always_inline)) { return page >= 0 && page < a.c.pages; };
    u4 k[2][KC];
    VT v[8];
    float ks[SC], vs[SC];
    unsigned mask = 0;                       // of the lane's 8 positions, those that are there
    bool some = false, all = false;          // of the tile's (uniform)
    // FAST: the four groups of 8 positions of the tile to be requested next: slot, place in the page, and the page, which comes through the scalar cache, a tile
    // ahead: a wait for it is none for codes under way.
    typedef const int32_t __attribute__((address_space(4))) *Entries;
    const Entries entries = (Entries)(uintptr_t)table;
    unsigned slot_at[4], off_at[4];
    int page_at[4];
    auto set = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned t = (unsigned)t0 * TP + 8 * i;
            slot_at[i] = t / page_size;
            off_at[i] = t - slot_at[i] * page_size;
            page_at[i] = entries[min(slot_at[i], last_slot)];
        }
    };
    auto advance = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            slot_at[i] += a.step_slots;
            off_at[i] += a.step_rest;
            if (off_at[i] >= page_size) { off_at[i] -= page_size; ++slot_at[i]; }
            page_at[i] = entries[min(slot_at[i], last_slot)];
        }
    };
    // one of two or four numbers
    auto pick = [&](bool one, int64_t x, int64_t y) __attribute__((always_inline)) { return one ? x : y; };
    auto by_group = [&](int group, int64_t x0, int64_t x1, int64_t x2, int64_t x3) __attribute__((always_inline)) {
        return group & 2 ? group & 1 ? x3 : x2 : group & 1 ? x1 : x0;
    };
    int64_t v_off = 0, s_off = 0;            // where the lane's rows of V, and its scales, of the tile requested next begin
    bool v_ok = false;
    // (a position beyond the length has a wrapped difference, too large for the range)
    auto there = [&](unsigned t) __attribute__((always_inline)) { return t - (unsigned)first < (unsigned)(len - first); };
    auto load = [](const auto *p) __attribute__((always_inline)) {
        if constexpr (LINES) return __builtin_nontemporal_load(p);
        else return *p;
    };
    auto load_k = [&](int x, int n, const char *row) __attribute__((always_inline)) {
        if constexpr (LINES) {
#pragma unroll
            for (int h = 0; h < KC / 2; ++h) k[x][2 * h + n] = load((const u4 *)(row + min(128 * h + 32 * g + 16 * (r16 >> 3), a.d - 16)));
        } else {
            k[x][0] = load((const u4 *)(row + min(16 * g, a.d - 16)));
        }
    };
    // not FAST: a lane finds one of the tile's 32 rows, the others ask it
    int64_t row_off = 0;
    float row_ks = 0.f, row_vs = 0.f;
    unsigned row_mask = 0;
    auto row_of = [&](int row) __attribute__((always_inline)) {
        const int lo = __shfl((int)row_off, row, 64), hi = __shfl((int)(row_off >> 32), row, 64);
        return (int64_t)(((uint64_t)(unsigned)hi << 32) | (unsigned)lo);
    };
    auto request_k = [&](int i) __attribute__((always_inline)) {
        const unsigned start = (unsigned)(t0 + i) * TP;
        if constexpr (FAST) {
            int64_t row[4], scale[4];
            bool ok = true, ok_at[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                ok_at[q] = in_pool(page_at[q]);
                ok &= ok_at[q];
                row[q] = page_at[q] * a.c.page + (int64_t)off_at[q] * a.c.position;
                scale[q] = page_at[q] * scale_page + a.s.by_block.of(off_at[q]);
            }
            advance();
            v_off = by_group(g, row[0], row[1], row[2], row[3]);
            s_off = by_group(g, scale[0], scale[1], scale[2], scale[3]);
            all = ok && start >= (unsigned)first && start + TP <= (unsigned)len;
            int64_t k_off[KR][2];
            bool k_ok[KR];
#pragma unroll
            for (int n = 0; n < KR; ++n) {
                const bool odd = r16 >> 2 & 1;
                k_off[n][0] = (LINES ? pick(odd, row[2 * n + 1], row[2 * n]) : by_group(r16 >> 2, row[0], row[1], row[2], row[3])) + (r16 & 3) * a.c.position;
                k_off[n][1] = k_off[n][0] + 4 * a.c.position;
            }
            if (!all) {
                // a row that is not there is replaced by one that is, so that as many requests are under way for every tile; where there is none, by some place of the pool
                v_ok = by_group(g, ok_at[0], ok_at[1], ok_at[2], ok_at[3]) != 0;
                uint64_t lanes[KR][2];
                int64_t other = 0;
#pragma unroll
                for (int n = 0; n < KR; ++n) {
                    const bool odd = r16 >> 2 & 1;
                    k_ok[n] = (LINES ? pick(odd, ok_at[2 * n + 1], ok_at[2 * n]) : by_group(r16 >> 2, ok_at[0], ok_at[1], ok_at[2], ok_at[3])) != 0;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        lanes[n][x] = __ballot(k_ok[n] & there(start + k_row(n) + 4 * x));
                        if (lanes[n][x]) {
                            const int from = __ffsll((long long)lanes[n][x]) - 1;
                            other = (int64_t)(((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(k_off[n][x] >> 32), from) << 32) |
                                              (unsigned)__builtin_amdgcn_readlane((int)k_off[n][x], from));
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < KR; ++n)
#pragma unroll
                    for (int x = 0; x < 2; ++x) k_off[n][x] = (k_ok[n] & there(start + k_row(n) + 4 * x)) ? k_off[n][x] : other;
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int n = 0; n < KR; ++n) load_k(x, n, Kh + k_off[n][x]);
        } else {
            const unsigned t = start + (lane & 31), slot = t / page_size, off = t - slot * page_size;
            const int page = there(t) ? table[slot] : -1;
            const bool ok = in_pool(page);
            row_mask = (unsigned)__ballot(ok);
            row_off = ok ? page * a.c.page + off * a.c.position : 0;
            row_ks = row_vs = 0.f;
            if (ok) {
                const int64_t s = page * scale_page + a.s.by_block.of(off);
                row_ks = Ks[s]; row_vs = Vs[s];
            }
            if (row_mask != ~0u) {           // a position that is not there is replaced by one that is: what storage without a meaning holds reaches nothing
                const int64_t other = row_of(row_mask ? __ffs((int)row_mask) - 1 : 0);
                if (!ok) row_off = other;
            }
            if (row_mask) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int n = 0; n < KR; ++n) load_k(x, n, Kh + row_of(k_row(n) + 4 * x));
            }
        }
    };
    auto request_v = [&](int i) __attribute__((always_inline)) {
        const unsigned start = (unsigned)(t0 + i) * TP, tv = start + v_row;
        if constexpr (FAST) {
            mask = 0xff; some = true;
            int64_t row[8], of = s_off;
#pragma unroll
            for (int j = 0; j < 8; ++j) row[j] = v_off + j * a.c.position;
            if (!all) {
                // rows from lo to hi are there; the others are replaced by the nearest of them, or by another lane's
                int lo = max(0, first - (int)tv), hi = (int)min((int64_t)7, (int64_t)len - 1 - tv);
                const bool any = v_ok & (lo <= hi);
                const uint64_t lanes = __ballot(any);
                some = lanes != 0;
                mask = any ? (0xffu << lo) & (0xffu >> (7 - hi)) : 0u;
                int64_t at = v_off + lo * a.c.position;
                const int from = some ? __ffsll((long long)lanes) - 1 : 0;
                const int low = __builtin_amdgcn_readlane((int)at, from), high = __builtin_amdgcn_readlane((int)(at >> 32), from);
                at = any ? v_off : some ? (int64_t)(((uint64_t)(unsigned)high << 32) | (unsigned)low) : 0;
                lo = any ? lo : 0;
                hi = any ? hi : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) row[j] = at + min(max(j, lo), hi) * a.c.position;
                of = any ? of : 0;
            }
            // (one sequence of requests for both kinds of tiles: the compiler's waits are by count, and by the shortest way)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = load((const VT *)(Vh + row[j]));
            ks[0] = Ks[of]; vs[0] = Vs[of];
        } else {
            mask = row_mask >> v_row & 0xffu;
            some = row_mask != 0;
            all = row_mask == ~0u;
            if (some) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = *(const VT *)(Vh + row_of(v_row + j));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) { ks[j] = __shfl(row_ks, v_row + j, 64); vs[j] = __shfl(row_vs, v_row + j, 64); }
        }
    };
    // ---- query rows: row r of the key head is beam r / group, head kvh * group + r % group; 8 elements from column k_col(c) + 8 h on a piece ----
    u4 q[RG][QP][KC][2];
    float slope[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        const int r = row0 + 16 * rg + r16;
        const bool here = 16 * rg + r16 < a.rows && r < a.R, f32 = QP > 1 && a.dtype == EL_F32;
        const int head = kvh * a.group + r % a.group, es = f32 ? 4 : 2;
        const char *const p = a.queries + (b * a.beam + r / a.group) * a.query_stride + (int64_t)head * a.d * es;
#pragma unroll
        for (int c = 0; c < 2 * KC; ++c) {
            const int col = k_col(c >> 1) + 8 * (c & 1);
            u4 w0 = u4{0, 0, 0, 0}, w1 = w0;
            if (here && col < a.d) {
                w0 = *(const u4 *)(p + col * es);
                if (f32) w1 = *(const u4 *)(p + col * es + 16);
            }
            if constexpr (QP == 1) {
                q[rg][0][c >> 1][c & 1] = w0;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned w = w0[i];        // (a bit cast of a vector's element itself takes element 0 whatever the index)
                    const h2 half = __builtin_bit_cast(h2, w);
                    float u = f32 ? __uint_as_float(i < 2 ? w0[2 * i] : w1[2 * i - 4]) : a.dtype == EL_F16 ? (float)half[0] : __uint_as_float(w << 16);
                    float v = f32 ? __uint_as_float(i < 2 ? w0[2 * i + 1] : w1[2 * i - 3]) : a.dtype == EL_F16 ? (float)half[1] : __uint_as_float(w & 0xffff0000u);
#pragma unroll
                    for (int n = 0; n < QP; ++n) {
                        const unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{u, v}, b2));
                        const float x = __uint_as_float(h << 16), y = __uint_as_float(h & 0xffff0000u);
                        q[rg][n][c >> 1][c & 1][i] = h;
                        u = fabsf(x) == INFINITY ? 0.f : u - x;      // (an infinity is one in the first part)
                        v = fabsf(y) == INFINITY ? 0.f : v - y;
                    }
                }
            }
        }
        slope[rg] = here && a.slopes ? a.slopes[head] : 0.f;
    }

    if (nt > 0) {
        if constexpr (FAST) set();
        request_k(0);
        request_v(0);
        // (the queries are waited for here: a wait for them inside the loop would be one for all that is under way)
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
#pragma unroll
            for (int n = 0; n < QP; ++n)
#pragma unroll
                for (int c = 0; c < 2 * KC; ++c) asm volatile("" : "+v"(q[rg][n][c >> 1][c & 1]));
            asm volatile("" : "+v"(slope[rg]));
        }
    }

    f4 acc[RG][DT16];
    float m[RG], l[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        m[rg] = -INFINITY; l[rg] = 0.f;
#pragma unroll
        for (int t = 0; t < DT16; ++t) acc[rg][t] = f4{0.f, 0.f, 0.f, 0.f};
    }

    f4 s[RG][2];
    auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if constexpr (LINES) {           // row r16's chunks 2 h and 2 h + 1: half of the lanes have the one of it and the other's of row r16 ^ 8
#pragma unroll
                for (int h = 0; h < KC / 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k0 = (int)k[x][2 * h][e], k1 = (int)k[x][2 * h + 1][e];
                        k[x][2 * h][e] = (unsigned)__builtin_amdgcn_update_dpp(k0, k1, kRor8, 0xf, 0xc, false);
                        k[x][2 * h + 1][e] = (unsigned)__builtin_amdgcn_update_dpp(k1, k0, kRor8, 0xf, 0x3, false);
                    }
            }
#pragma unroll
            for (int rg = 0; rg < RG; ++rg) s[rg][x] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned w0 = k[x][c][2 * h], w1 = k[x][c][2 * h + 1];
                    const u4 kk = {KN::template two<false>(w0), KN::template two<true>(w0), KN::template two<false>(w1), KN::template two<true>(w1)};
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                        for (int p = QP - 1; p >= 0; --p) s[rg][x] = Mma<BF16>::s16(kk, q[rg][p][c][h], s[rg][x]);
                }
        }
    };
    auto sums = [&](int i, bool whole_tile) __attribute__((always_inline)) {
        const int dist = (int)((unsigned)(len - 1) - ((unsigned)(t0 + i) * TP + v_row));         // of the lane's first position
        const unsigned mask_now = mask;
        // ---- softmax: lane (g, r16) holds positions 8 g + 4 x + e of row r16 ----
        // (the largest score is taken from the others before they become powers of two: what scores have in common takes no digits from their
        // distances)
        u4 pp[RG][NP];
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
            float p[8], mx;
            const bool plain = FAST && whole_tile && !a.shaped;
            const float v1 = mask_now ? vs[0] : 0.f;                 // (what stands for the scale of positions that are not there reaches nothing)
            if (plain) {
                mx = s[rg][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[rg][j >> 2][j & 3]);
                mx *= ks[0];
            } else {
                mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = s[rg][j >> 2][j & 3] * ks[FAST ? 0 : j];
                    if (a.shaped) {
                        p[j] *= a.product;
                        if (a.softcap > 0.f) p[j] = a.softcap * tanhf(p[j]);
                        if (a.slopes) p[j] = fmaf(-slope[rg], (float)(dist - j), p[j]);
                    }
                    if (!((mask_now >> j) & 1)) p[j] = -INFINITY;
                    mx = fmaxf(mx, p[j]);
                }
            }
            if (__ballot(mx > m[rg])) {
                mx = fmaxf(m[rg], max_over_groups(mx));
                const float f = m[rg] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[rg] - mx) * a.unit);
                l[rg] *= f;
#pragma unroll
                for (int t = 0; t < DT16; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[rg][t][e] *= f;
                m[rg] = mx;
            }
            const float ref = m[rg] == -INFINITY ? 0.f : m[rg];
            if (plain) {
                const float k1 = ks[0];
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = fmaf(s[rg][j >> 2][j & 3], k1, -ref);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] -= ref;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(p[j] * a.unit);
                l[rg] += p[j];
                p[j] *= FAST ? v1 : vs[j];
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                float u = p[2 * y], x = p[2 * y + 1];
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    const unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{u, x}, b2));
                    pp[rg][n][y] = h;
                    u -= __uint_as_float(h << 16); x -= __uint_as_float(h & 0xffff0000u);
                }
            }
        }
        // ---- weighted sum ----
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            auto column = [&](auto I) __attribute__((always_inline)) {
                constexpr int j = decltype(I)::value;
                u4 vv;
#pragma unroll
                for (int y = 0; y < 4; ++y) vv[y] = VN::template of_two<j>(VB::at(v[2 * y], c), VB::at(v[2 * y + 1], c));
#pragma unroll
                for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                    for (int n = NP - 1; n >= 0; --n) acc[rg][4 * c + j] = Mma<true>::s16(vv, pp[rg][n], acc[rg][4 * c + j]);
            };
            column(std::integral_constant<int, 0>{});
            column(std::integral_constant<int, 1>{});
            column(std::integral_constant<int, 2>{});
            column(std::integral_constant<int, 3>{});
        }
    };
    // Codes of the next tile's keys are requested when this one's have been multiplied, those of its values when this one's have.  (The last tile apart: on every way
    // through the loop as many requests follow one another, and the compiler's waits are by count.)
    if (nt > 0) {
        int i = 0;
#pragma unroll 1
        for (; i + 1 < nt; ++i) {
            scores();
            const bool none = !some, whole_tile = all;
            if constexpr (FAST) request_k(i + 1);
            if (!none) sums(i, whole_tile);
            if constexpr (!FAST) request_k(i + 1);
            request_v(i + 1);
        }
        scores();
        if (some) sums(i, all);
    }

    int at = lane, group = a.group;
    asm volatile("" : "+v"(at), "+s"(group));     // (as above: worked out anew, instead of being held over the tiles)
    const int ar = at & 15, ag = at >> 4;
    const bool whole = pieces == 1;
    const int64_t slot = ((int64_t)(span + st.b) * units + unit) * a.rows;
    const int waves = a.waves;
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) l[rg] = sum_over_groups(l[rg]);
    // columns (4 g + e) DP / 16 + 4 jq .. + 3 of the row are item e KC + jq of its lane
    auto item = [&](int rg, int t) __attribute__((always_inline)) {
        const int e = t / KC, jq = t % KC;
        return f4{acc[rg][4 * jq][e], acc[rg][4 * jq + 1][e], acc[rg][4 * jq + 2][e], acc[rg][4 * jq + 3][e]};
    };
    f4 *const X = (f4 *)shared;                                      // [wavefront][rg][item][lane]
    float2 *const ml = (float2 *)(shared + waves * (RG * DP * 64));  // [wavefront][rg][row]
    if (waves > 1) {
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
            if (ag == 0) ml[(wave * RG + rg) * 16 + ar] = float2{m[rg], l[rg]};
#pragma unroll
            for (int t = 0; t < ITEMS; ++t) X[((wave * RG + rg) * ITEMS + t) * 64 + at] = item(rg, t);
        }
        __syncthreads();
    }
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        const int rb = 16 * rg + ar, r = row0 + rb;
        float M = m[rg], L = l[rg];
        // (a wavefront without a position: sum 0.  A NaN score leaves its maximum at -inf and its sum at NaN, which stays)
        auto factor = [&](float mk) __attribute__((always_inline)) { return mk == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mk - M) * a.unit); };
        if (waves > 1) {
            M = -INFINITY; L = 0.f;
#pragma unroll 1
            for (int n = 0; n < waves; ++n) M = fmaxf(M, ml[(n * RG + rg) * 16 + ar].x);
#pragma unroll 1
            for (int n = 0; n < waves; ++n) { const float2 x = ml[(n * RG + rg) * 16 + ar]; L += factor(x.x) * x.y; }
        }
        if (rb >= a.rows || r >= a.R) continue;
        // no score, or none above -inf: 0, unless there is a NaN among them
        const bool empty = whole && M == -INFINITY && !(L != L);
        const int64_t out_row = (b * a.beam + r / group) * a.heads + kvh * group + r % group;
        if (ag == 0 && wave == 0) {
            if (!whole) a.part_ml[slot + rb] = float2{M, L};
            else if (a.lse) a.lse[out_row] = empty ? -INFINITY : fmaf(M, a.natural, __builtin_amdgcn_logf(L) * kLn2);
        }
        const float inv = whole ? 1.f / L : 1.f;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            const int col = (4 * ag + t / KC) * (DP / 16) + 4 * (t % KC);
            if (col >= a.d || (t & (waves - 1)) != wave) continue;   // (each wavefront finishes every waves-th item)
            f4 o = item(rg, t);
            if (waves > 1) {
                o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int n = 0; n < waves; ++n) {
                    const float f = factor(ml[(n * RG + rg) * 16 + ar].x);
                    const f4 x = X[((n * RG + rg) * ITEMS + t) * 64 + at];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] += f * x[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = empty ? 0.f : o[e] * inv;
            if (whole) store4(a.out, out_row * a.d + col, a.out_dtype, o);
            else *(f4 *)(a.part_o + (slot + rb) * a.d + col) = o;
        }
    }
    if (!a.spans) return;
    st.at += nt;
    if (st.aligned || st.at >= st.end) return;
    st.before += tiles;
    ++st.b;
    }
}

bool is_fast(const el_attn_pages8 &c) { return c.page_size % 8 == 0 && c.block % 8 == 0; }

template <class Fn>
void with_form8(const el_attn_pages8 &c, int dtype, int row_groups, Fn fn)
{
    auto parts = [&](auto fmt, auto width, auto rg) {
        constexpr int FMT = decltype(fmt)::value, DP = decltype(width)::value, RG = decltype(rg)::value;
        if (!is_fast(c)) { if constexpr (RG == 1) fn(Form8<FMT, DP, 1, EL_F32, false>{}); }
        else if constexpr (DP < 256 || RG == 1) {
            if (dtype == EL_F32) fn(Form8<FMT, DP, RG, EL_F32, true>{});
            else if (dtype == EL_F16) fn(Form8<FMT, DP, RG, EL_F16, true>{});
            else fn(Form8<FMT, DP, RG, EL_BF16, true>{});
        }
    };
    auto rows = [&](auto fmt, auto width) {
        if (row_groups == 1) parts(fmt, width, std::integral_constant<int, 1>{});
        else parts(fmt, width, std::integral_constant<int, 2>{});
    };
    auto widths = [&](auto fmt) {
        if (c.d_head <= 64) rows(fmt, std::integral_constant<int, 64>{});
        else if (c.d_head <= 128) rows(fmt, std::integral_constant<int, 128>{});
        else rows(fmt, std::integral_constant<int, 256>{});
    };
    if (c.format == EL_E4M3) widths(std::integral_constant<int, EL_E4M3>{});
    else widths(std::integral_constant<int, EL_INT8>{});
}

AttendPlan plan_attend8(const el_attn_pages8 &c, int dtype, int heads, int B, int beam, int n)
{
    const int R = beam * (heads / c.kv_heads);
    SpanForm form{};
    form.padded = c.d_head <= 64 ? 64 : c.d_head <= 128 ? 128 : 256;
    // two groups of rows share a tile's codes; 256 columns leave no registers for them, and without FAST there is one form
    form.row_groups = R <= 16 || !is_fast(c) || form.padded == 256 ? 1 : 2;
    form.tile = TP;
    with_form8(c, dtype, form.row_groups, [&](auto f) { form.per_cu = f.PER_CU; form.most = f.WAVES; form.lds = f.LDS; });
    AttendPlan p = plan_spans(form, R, c.kv_heads, c.d_head, form.padded, c.head_stride, B, n);
    if (p.waves == 1) p.lds = 0;
    return p;
}

bool valid_types(int32_t dtype, int32_t out_dtype)
{
    return (dtype == EL_F32 || dtype == EL_F16 || dtype == EL_BF16) && (out_dtype == EL_F32 || out_dtype == dtype);
}

} // namespace
} // namespace el

extern "C" size_t el_attn_quantized_workspace_bytes(const el_attn_pages8 *cache, int32_t dtype, int32_t out_dtype, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    if (el::check_pages8(cache) != EL_OK || !el::valid_types(dtype, out_dtype) || !el::valid_sizes(cache->kv_heads, heads, B, beam, n)) return 0;
    return el::plan_attend8(*cache, dtype, heads, B, beam, n).workspace;
}

extern "C" el_status el_attn_quantized_attend(const el_attn_pages8 *cache, int32_t dtype,
                                              const int32_t *table, int64_t table_stride, int32_t table_pages, const int32_t *lengths,
                                              const void *queries, int64_t query_stride, int32_t heads, const el_attn_score_rule *rule,
                                              void *out, int32_t out_dtype, float *lse, int32_t B, int32_t beam, int32_t n,
                                              void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (const el_status st = check_pages8(cache); st != EL_OK) return st;
    if (!valid_types(dtype, out_dtype)) return EL_ERR_UNSUPPORTED;
    const AttendOperands o{table, table_stride, table_pages, lengths, queries, query_stride, heads, dtype, rule, out, out_dtype, lse, B, beam, n};
    if (const el_status st = check_attend(o, cache->kv_heads, cache->d_head, cache->page_size); st != EL_OK) return st;
    const AttendPlan p = plan_attend8(*cache, dtype, heads, B, beam, n);
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return EL_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 15) return EL_ERR_INVALID_ARG;
    }
    Attend8Args a{};
    (AttendArgs &)a = attend_args(o, page_view8(*cache, table, table_stride, table_pages), cache->kv_heads, cache->d_head, lse, out, p, workspace);
    a.s = scale_view(*cache);
    a.dtype = dtype;
    a.step_slots = TP / cache->page_size;
    a.step_rest = TP % cache->page_size;
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    with_form8(*cache, dtype, p.row_groups, [&](auto f) {
        hipLaunchKernelGGL((k_coded_attend<decltype(f)>), dim3((unsigned)p.grid), dim3(64 * p.waves), p.lds, s, a);
    });
    if (hipGetLastError() != hipSuccess) return EL_ERR_HIP;
    return p.spans ? launch_join(a, p, s) : EL_OK;
}
