// Attention of one new token per query row over a sequence's pages of projected keys and values.
//
//   s_t = scale q.K_t (capped, biased by distance),  out = sum_t softmax(s)_t V_t,  lse = log sum_t exp s_t
//
// over the positions that are there: below the length, inside the window, in a page of the pool.
//
// Bound by HBM: every key and value is read once and used by the query rows of its sequence that share the key head (beam x
// heads / kv_heads of them, a handful), 2 flops a byte and row.  The kernel is built to keep that stream running:
//   - A wavefront works alone on tiles of 32 positions (16 in fp32) of one sequence and key head, with a ring of tiles in LDS that
//     is filled by direct requests (16 bytes a lane, no registers in flight) and waited for by count.  The page numbers
//     of a tile are requested the same way, a ring's depth ahead, so that no request waits for the table.
//   - Scores and weighted sum are matrix products, S^T = K Q^T and O^T += V^T P^T, with up to 16 query rows as columns.  S^T leaves
//     the matrix unit with 4 neighbouring positions of one row in a lane; taken as the 8 inner indices of the second product (two
//     groups of 16 positions), P never leaves the registers, and V's columns come from LDS transposed (ds_read_b64_tr_b16).
//   - The running maximum and sum of the softmax are kept per wavefront; k_attend_join joins the pieces of a sequence.
// Work: paged_spans.h.
#include <type_traits>
#include "paged_spans.h"

namespace el {
namespace {

// Keys and values pass the caches by: between two reads of a layer's cache lie those of all others.  us, inputs that are in no cache, kept in
// them / passed by: 512 continuations of up to 256 positions 63 / 57, 64 sequences of 1024 to 4096 135 / 120, two of up to 131072 178 / 161.
// (Two blocks of rows that read the same, more than 32 rows a key head, lose 3 %; a cache that the memory-side cache holds from call to call 4 to 9 %.)
__device__ __forceinline__ void request16(unsigned lds_addr, const char *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" :: "s"(lds_addr), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void request4(unsigned lds_addr, const int32_t *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(lds_addr), "v"(from) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_requests() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// Row `row` of a tile keeps its chunk c of 16 bytes at c ^ swizzle(row): operand reads of 16 rows at one chunk, and the transposing
// reads of 16 rows at two, then spread over all banks.
template <int ROWB> __device__ __forceinline__ int swizzle(int row) { return ROWB >= 256 ? row & 15 : (row >> 1) & 7; }

// The product with 16 inner indices, 4 of them in a lane.
template <bool BF16> __device__ __forceinline__ f4 k16(s4 a, u2 b, f4 c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s4, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(h4, a), __builtin_bit_cast(h4, b), c, 0, 0, 0);
}

// What a wavefront is built for: storage type, d_head padded, query rows in groups of 16.
template <int DT_, int DP_, int RG_> struct Form {
    static constexpr int DT = DT_, DP = DP_, RG = RG_;
    static constexpr bool F32 = DT == EL_F32, BF16 = DT == EL_BF16;
    static constexpr int ES = F32 ? 4 : 2, ROWB = DP * ES;
    static constexpr int TP = F32 || DP == 256 ? 16 : 32;            // positions of a tile
    static constexpr int TILEB = TP * ROWB;                          // bytes of a tile's keys
    // Tiles in the ring: one used, one under way.  More wavefronts a compute unit beat deeper rings: with three and four tiles 64 sequences of
    // 1024 to 4096 positions (8 key heads of 128) take 154 and 200 us for 136, 512 of up to 256 (16 of 64) 65 and 80 for 54.
    static constexpr int NS = 2;
    static constexpr int RING = NS * 2 * TILEB, LDS = RING + NS * 256;             // of a wavefront: tiles, page numbers
    static constexpr int ROOM = 163840 / LDS, MOST = RG == 2 ? 8 : 12;             // by LDS; by registers
    static constexpr int PER_CU = ROOM < MOST ? ROOM : MOST;                       // wavefronts that a compute unit holds
    static constexpr int WAVES = PER_CU >= 8 ? 8 : PER_CU >= 4 ? 4 : 2;            // of a workgroup, at most
};

// NP: parts of a probability (launch_attend).
template <class F, int NP>
__global__ void __launch_bounds__(64 * F::WAVES, (F::PER_CU + 3) / 4) k_attend(const AttendArgs a)
{
    constexpr bool F32 = F::F32, BF16 = F::BF16;
    constexpr int DT = F::DT, DP = F::DP, RG = F::RG, ES = F::ES, TP = F::TP, ROWB = F::ROWB, NS = F::NS, TILEB = F::TILEB;
    constexpr int CPR = ROWB / 16, NI = TILEB / 1024, RPI = 64 / CPR, PENDING = (NS - 1) * (2 * NI + 1), DT16 = DP / 16;
    constexpr int QC = F32 ? DP / 16 : DP / 32;                      // pieces of 16 bytes of a query row that a lane holds
    // P in 16 bits: parts that add up to it.  fp16: times 2^15, which keeps the low parts of small ones out of the subnormal numbers (what is lost
    // there is 2^-40 of the largest at most).
    constexpr float PARTS = DT == EL_F16 ? 32768.f : 1.f;
    extern __shared__ __attribute__((aligned(1024))) char shared[];  // [wavefront] ring of tiles; then [wavefront] page numbers of NS tiles

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char *const ring = shared + wave * F::RING;
    int *const Tb = (int *)(shared + a.waves * F::RING + wave * (NS * 256));
    const int units = a.kv_heads * a.row_blocks;
    int span = blockIdx.x / units, unit = blockIdx.x - span * units;
    if (a.near && (span / kDies + 1) * kDies * units <= (int)gridDim.x) {            // workgroups go round the dies: a die takes a span's units
        const int first = span / kDies * kDies, i = blockIdx.x - first * units;
        span = first + i % kDies;
        unit = i / kDies;
    }
    const int kvh = unit % a.kv_heads, row0 = unit / a.kv_heads * a.rows;
    EL_LDS(char) *const lds = (EL_LDS(char) *)ring;
    const unsigned lds_at = (unsigned)(uintptr_t)lds, tb_at = (unsigned)(uintptr_t)(EL_LDS(int) *)Tb;
    const int chunks = a.d * ES / 16;
    if (chunks < CPR) {                     // columns beyond d_head are never requested: zeros, which a query's zeros meet
        for (int i = threadIdx.x & 63; i < F::RING / 16; i += 64) *(u4 *)(ring + i * 16) = u4{0, 0, 0, 0};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const char *const Kh = a.c.K + kvh * a.c.head;
    const int64_t k_to_v = a.c.V - a.c.K;

    Start st{span, 0, 0, 0, 1, false};
    if (a.spans && !find_span(a, span, TP, st)) return;
    // the pieces of this span: the tiles of one sequence after the other
    for (;;) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));          // (what follows from it is worked out anew for a piece, instead of being held over all of them)
    const int r16 = lane & 15, g = lane >> 4;
    const int64_t b = st.b;
    // query rows: row r of the key head is beam r / group, head kvh * group + r % group
    u4 q[RG][QC];
    float slope[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        const int r = row0 + 16 * rg + r16;
        const bool here = 16 * rg + r16 < a.rows && r < a.R;
        const int head = kvh * a.group + r % a.group;
        const char *p = a.queries + (b * a.beam + r / a.group) * a.query_stride + (int64_t)head * a.d * ES;
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            q[rg][c] = u4{0, 0, 0, 0};
            if (here && (4 * c + g) * 16 < a.d * ES) q[rg][c] = *(const u4 *)(p + (4 * c + g) * 16);
        }
        slope[rg] = here && a.slopes ? a.slopes[head] : 0.f;
    }
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

    f4 acc[RG][DT16];
    float m[RG], l[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        m[rg] = -INFINITY; l[rg] = 0.f;
#pragma unroll
        for (int t = 0; t < DT16; ++t) acc[rg][t] = f4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t *const table = a.c.table + b * a.c.table_stride;
    auto slot_of = [&](int i) __attribute__((always_inline)) { return (int)((unsigned)i % NS); };
    auto position = [&](int i) __attribute__((always_inline)) { return (int64_t)(t0 + i) * TP + (lane & (TP - 1)); };
    auto request_pages = [&](int i) __attribute__((always_inline)) {
        const int64_t last = (int64_t)len - 1, t = position(i) < last ? position(i) : last;
        request4(tb_at + slot_of(i) * 256, table + (unsigned)t / (unsigned)a.c.page_size);
    };
    // Requests tile i; returns which of its positions are there.  One that is not is replaced by one that is: what storage without
    // a meaning holds reaches nothing.
    auto request_tile = [&](int i) __attribute__((always_inline)) -> unsigned {
        const int64_t t = position(i);
        const unsigned slot = (unsigned)(t < len ? t : 0) / (unsigned)a.c.page_size;
        const int page = Tb[slot_of(i) * 64 + lane];
        const bool valid = t >= first && t < len && page >= 0 && page < a.c.pages;
        constexpr unsigned ALL = TP == 32 ? 0xffffffffu : 0xffffu;
        const unsigned mask = (unsigned)__ballot(valid) & ALL;
        int64_t off = valid ? page * a.c.page + (t - (int64_t)slot * a.c.page_size) * a.c.position : 0;
        if (mask != ALL) {
            const int some = mask ? __ffs((int)mask) - 1 : 0;
            const int lo = __builtin_amdgcn_readlane((int)off, some), hi = __builtin_amdgcn_readlane((int)(off >> 32), some);
            if (!valid) off = (int64_t)(((uint64_t)(unsigned)hi << 32) | (unsigned)lo);
        }
        const unsigned at = lds_at + slot_of(i) * (2 * TILEB);
        int have = chunks;
        asm volatile("" : "+s"(have));      // (compared anew for a tile: NI masks of lanes held over the loop are more registers than there are)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int row = j * RPI + lane / CPR, c = (lane % CPR) ^ swizzle<ROWB>(row);
            const int lo = __shfl((int)off, row, 64), hi = __shfl((int)(off >> 32), row, 64);
            const char *from = Kh + (int64_t)(((uint64_t)(unsigned)hi << 32) | (unsigned)lo) + c * 16;
            if (c < have) {                 // (at least the first chunk of a row: the instruction is issued, and counted, always)
                request16(at + j * 1024, from);
                request16(at + TILEB + j * 1024, from + k_to_v);
            }
        }
        return mask;
    };

    if (nt > 0) {
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) request_pages(i);
    }
    // (in registers before the first tile is requested: a wait of the compiler's for them would wait for all that is under way)
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
#pragma unroll
        for (int c = 0; c < QC; ++c) asm volatile("" : "+v"(q[rg][c]));
        asm volatile("" : "+v"(slope[rg]));
    }
    unsigned here[NS];
    if (nt > 0) {
        wait_requests<0>();
#pragma unroll
        for (int i = 0; i < NS - 1; ++i) {
            request_pages(i + NS - 1);
            here[i] = 0;
            if (i < nt) here[i] = request_tile(i);
        }
    }
    for (int i = 0; i < nt; ++i) {
        // Requests come back in order.  Behind the pages of tile i + NS - 1, and behind tile i, exactly NS - 1 tiles and their pages
        // have been requested; at the end of the span, where there are fewer, everything is waited for.
        request_pages(i + 2 * NS - 2);
        here[NS - 1] = 0;
        if (i + NS - 1 < nt) {
            wait_requests<PENDING>();
            here[NS - 1] = request_tile(i + NS - 1);
            wait_requests<PENDING>();
        } else {
            wait_requests<0>();
        }
        const unsigned mask = here[0];
#pragma unroll
        for (int k = 0; k < NS - 1; ++k) here[k] = here[k + 1];
        if (mask == 0) continue;
        const EL_LDS(char) *const Kt = lds + slot_of(i) * (2 * TILEB), *const Vt = Kt + TILEB;
        const int dist0 = len - 1 - (t0 + i) * TP;             // of the tile's first position

        // ---- scores ----
        constexpr int NA = TP / 16;
        f4 s[RG][NA];
#pragma unroll
        for (int x = 0; x < NA; ++x) {
            u4 k[QC];
#pragma unroll
            for (int c = 0; c < QC; ++c) k[c] = *(const EL_LDS(u4) *)(Kt + (16 * x + r16) * ROWB + (((4 * c + g) ^ swizzle<ROWB>(r16)) << 4));
            // fp32: four sums instead of one of d / 4 instructions, each of which rounds.  The error of a result against fp64 falls from up to 2.3 times
            // to 1.1 times that of plain fp32 operations.  us, one sum / four: 250 sequences of 100 to 1000, 8 heads of 128 199 / 200, 4 of 256 423 / 413.
            constexpr int SUMS = F32 ? 4 : 1;
            f4 part[RG][SUMS];
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                for (int e = 0; e < SUMS; ++e) part[rg][e] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < QC; ++c)
#pragma unroll
                for (int rg = 0; rg < RG; ++rg) {
                    if constexpr (F32) {
                        const f4 kf = __builtin_bit_cast(f4, k[c]), qf = __builtin_bit_cast(f4, q[rg][c]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) part[rg][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[e], part[rg][e], 0, 0, 0);
                    } else {
                        part[rg][0] = Mma<BF16>::s16(k[c], q[rg][c], part[rg][0]);
                    }
                }
#pragma unroll
            for (int rg = 0; rg < RG; ++rg) {
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[rg][x][e] = (part[rg][0][e] + part[rg][1][e]) + (part[rg][2][e] + part[rg][3][e]);
                } else {
                    s[rg][x] = part[rg][0];
                }
            }
        }
        // ---- softmax: lane (g, r16) holds positions 16 x + 4 g + e of row r16 ----
        // (the largest score is taken from the others before they become powers of two: what scores have in common takes no digits from their
        // distances)
        const unsigned bits = mask >> (4 * g);
        const float unit = a.unit;
        float p[RG][NA][4];
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
#pragma unroll
            for (int x = 0; x < NA; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[rg][x][e] = s[rg][x][e];
            if (a.shaped) {
#pragma unroll
                for (int x = 0; x < NA; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[rg][x][e] *= a.product;
                if (a.softcap > 0.f) {
#pragma unroll
                    for (int x = 0; x < NA; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[rg][x][e] = a.softcap * tanhf(p[rg][x][e]);
                }
                if (a.slopes) {
#pragma unroll
                    for (int x = 0; x < NA; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[rg][x][e] = fmaf(-slope[rg], (float)(dist0 - 16 * x - 4 * g - e), p[rg][x][e]);
                }
            }
            if (mask != (TP == 32 ? 0xffffffffu : 0xffffu)) {
#pragma unroll
                for (int x = 0; x < NA; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!((bits >> (16 * x + e)) & 1)) p[rg][x][e] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int x = 0; x < NA; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, p[rg][x][e]);
            mx = fmaxf(m[rg], max_over_groups(mx));
            if (__ballot(mx > m[rg])) {
                const float f = m[rg] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[rg] - mx) * unit);
                l[rg] *= f;
#pragma unroll
                for (int t = 0; t < DT16; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[rg][t][e] *= f;
                m[rg] = mx;
            }
            const float ref = m[rg] == -INFINITY ? 0.f : m[rg];
#pragma unroll
            for (int x = 0; x < NA; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[rg][x][e] = __builtin_amdgcn_exp2f((p[rg][x][e] - ref) * unit);
                    l[rg] += p[rg][x][e];
                }
        }
        // ---- weighted sum ----
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < DT16; ++t) {
                    const int row = 4 * g + e;
                    const float v = *(const EL_LDS(float) *)(Vt + row * ROWB + (((4 * t + (r16 >> 2)) ^ swizzle<ROWB>(row)) << 4) + (r16 & 3) * 4);
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg) acc[rg][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[rg][0][e], acc[rg][t], 0, 0, 0);
                }
        } else {
            u4 pp[RG][NP];
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                for (int y = 0; y < 2 * NA; ++y) {
                    float u = p[rg][y >> 1][2 * (y & 1)] * PARTS, v = p[rg][y >> 1][2 * (y & 1) + 1] * PARTS;
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        if constexpr (BF16) {
                            const unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{u, v}, b2));
                            pp[rg][k][y] = h;
                            u -= __uint_as_float(h << 16); v -= __uint_as_float(h & 0xffff0000u);
                        } else {
                            const h2 h = __builtin_convertvector(f2{u, v}, h2);
                            pp[rg][k][y] = __builtin_bit_cast(unsigned, h);
                            u -= (float)h[0]; v -= (float)h[1];
                        }
                    }
                }
            const int row = 4 * g + (r16 >> 2);
#pragma unroll
            for (int t = 0; t < DT16; ++t) {
                const int at = row * ROWB + (((2 * t + ((r16 & 3) >> 1)) ^ swizzle<ROWB>(row)) << 4) + (r16 & 1) * 8;
                const s4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((EL_LDS(s4) *)(Vt + at));
                if constexpr (TP == 16) {
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                        for (int k = 0; k < NP; ++k) acc[rg][t] = k16<BF16>(v0, u2{pp[rg][k][0], pp[rg][k][1]}, acc[rg][t]);
                } else {
                    const s4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((EL_LDS(s4) *)(Vt + at + 16 * ROWB));
                    const u4 v = __builtin_bit_cast(u4, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                        for (int k = 0; k < NP; ++k) acc[rg][t] = Mma<BF16>::s16(v, pp[rg][k], acc[rg][t]);
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // every read of this slot is through before it is requested into
    }

    int waves = a.waves, w = wave;
    asm volatile("" : "+s"(waves), "+s"(w));                         // (as above)
    const bool whole = pieces == 1;
    const int64_t slot = ((int64_t)(span + st.b) * units + unit) * a.rows;
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) l[rg] = sum_over_groups(l[rg]);
    if (waves > 1) {
        // the wavefronts' results joined: each finishes every waves-th block of 16 columns
        float2 *const ml = (float2 *)Tb;                             // (of this wavefront: its own ring is through)
        f4 *const X = (f4 *)ring;
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
            if (g == 0) ml[16 * rg + r16] = float2{m[rg], l[rg]};
#pragma unroll
            for (int t = 0; t < DT16; ++t) X[(rg * DT16 + t) * 64 + lane] = acc[rg][t];
        }
        __syncthreads();
        float2 *const ml0 = (float2 *)(shared + waves * F::RING);
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
            float M = -INFINITY, L = 0.f;
            for (int k = 0; k < waves; ++k) M = fmaxf(M, ml0[k * (NS * 32) + 16 * rg + r16].x);
            // (a wavefront without a position: sum 0.  A NaN score leaves its maximum at -inf and its sum at NaN, which stays)
            auto factor = [&](int k) __attribute__((always_inline)) {
                const float mk = ml0[k * (NS * 32) + 16 * rg + r16].x;
                return mk == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mk - M) * a.unit);
            };
#pragma unroll
            for (int t = 0; t < DT16; ++t) acc[rg][t] = f4{0.f, 0.f, 0.f, 0.f};
            for (int k = 0; k < waves; ++k) {
                const float f = factor(k);
                L += f * ml0[k * (NS * 32) + 16 * rg + r16].y;
                const f4 *const Xk = (const f4 *)(shared + k * F::RING);
#pragma unroll
                for (int t = 0; t < DT16; ++t) {
                    if ((t & (waves - 1)) != w) continue;
                    const f4 x = Xk[(rg * DT16 + t) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[rg][t][e] += f * x[e];
                }
            }
            m[rg] = M; l[rg] = L;
        }
    }
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
        const int rb = 16 * rg + r16, r = row0 + rb;
        if (rb >= a.rows || r >= a.R) continue;
        const float M = m[rg], L = l[rg];
        // no score, or none above -inf: 0, unless there is a NaN among them
        const bool empty = whole && M == -INFINITY && !(L != L);
        const int64_t out_row = (b * a.beam + r / a.group) * a.heads + kvh * a.group + r % a.group;
        if (g == 0 && w == 0) {
            if (!whole) a.part_ml[slot + rb] = float2{M, L};
            else if (a.lse) a.lse[out_row] = empty ? -INFINITY : fmaf(M, a.natural, __builtin_amdgcn_logf(L) * kLn2);
        }
        // (a product with 1 / L: off by a step of fp32 where a division is by half of one.  Mended by two more operations an element, in fp32 results
        // alone, 512 continuations of up to 256 take 55.9 us, 55.2 so; 250 of 100 to 1000 in fp32, 8 heads of 128, 203 / 197)
        const float inv = (whole ? 1.f / L : 1.f) * (1.f / PARTS);
#pragma unroll
        for (int t = 0; t < DT16; ++t) {
            const int col = 16 * t + 4 * g;
            if (col >= a.d || (t & (waves - 1)) != w) continue;
            f4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = empty ? 0.f : acc[rg][t][e] * inv;
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

template <class Fn>
void with_form(int dtype, int padded, int row_groups, Fn fn)
{
    auto width = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (padded == 64) { if (row_groups == 1) fn(Form<DT, 64, 1>{}); else fn(Form<DT, 64, 2>{}); }
        else if (padded == 128) { if (row_groups == 1) fn(Form<DT, 128, 1>{}); else fn(Form<DT, 128, 2>{}); }
        else if (row_groups == 1) fn(Form<DT, 256, 1>{});
        else if constexpr (DT != EL_F32) fn(Form<DT, 256, 2>{});
    };
    if (dtype == EL_F32) width(std::integral_constant<int, EL_F32>{});
    else if (dtype == EL_F16) width(std::integral_constant<int, EL_F16>{});
    else width(std::integral_constant<int, EL_BF16>{});
}

AttendPlan plan_attend(const el_attn_pages &c, int heads, int B, int beam, int n)
{
    const int R = beam * (heads / c.kv_heads);
    SpanForm form{};
    form.padded = c.d_head <= 64 ? 64 : c.d_head <= 128 ? 128 : 256;
    // Two groups of rows share a tile's operand reads; in fp32 beyond 128 columns their registers do not suffice.  (Four, for more than 32
    // rows, gain nothing sure: 16 sequences of 1000 to 4096, 8 key heads of 128, 64 rows 75 us with two blocks of two / 70 with one of four,
    // 16 key heads of 64 51 / 55.)
    form.row_groups = R <= 16 || (c.dtype == EL_F32 && form.padded == 256) ? 1 : 2;
    with_form(c.dtype, form.padded, form.row_groups, [&](auto f) { form.tile = f.TP; form.per_cu = f.PER_CU; form.most = f.WAVES; form.lds = f.LDS; });
    const int64_t es = (int64_t)dtype_size(c.dtype);
    return plan_spans(form, R, c.kv_heads, c.d_head, form.padded * es, c.head_stride * es, B, n);
}

void launch_attend(const AttendArgs &a, const AttendPlan &p, int dtype, hipStream_t s)
{
    const dim3 grid((unsigned)p.grid);
    with_form(dtype, p.padded, p.row_groups, [&](auto f) {
        using F = decltype(f);
        // Parts of a probability in 16 bits: three hold its 24 bits, the products that they cost are mostly hidden behind HBM.  Two fp16 ones hold
        // 22, which a result in fp16 does not see: 16 sequences of 1000 to 4096, 32 rows on each of 4 key heads of 256, 61 us with two, 63 with three.
        if constexpr (F::F32) hipLaunchKernelGGL((k_attend<F, 1>), grid, dim3(64 * p.waves), p.lds, s, a);
        else if (F::BF16 || a.out_dtype == EL_F32) hipLaunchKernelGGL((k_attend<F, 3>), grid, dim3(64 * p.waves), p.lds, s, a);
        else if constexpr (!F::BF16) hipLaunchKernelGGL((k_attend<F, 2>), grid, dim3(64 * p.waves), p.lds, s, a);
    });
}

} // namespace
} // namespace el

extern "C" size_t el_attn_paged_workspace_bytes(const el_attn_pages *cache, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    if (el::check_pages(cache) != EL_OK || !el::valid_sizes(cache->kv_heads, heads, B, beam, n)) return 0;
    return el::plan_attend(*cache, heads, B, beam, n).workspace;
}

extern "C" el_status el_attn_paged_attend(const el_attn_pages *cache,
                                          const int32_t *table, int64_t table_stride, int32_t table_pages, const int32_t *lengths,
                                          const void *queries, int64_t query_stride, int32_t heads, const el_attn_score_rule *rule,
                                          void *out, int32_t out_dtype, float *lse, int32_t B, int32_t beam, int32_t n,
                                          void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace el;
    if (const el_status st = check_pages(cache); st != EL_OK) return st;
    const AttendOperands o{table, table_stride, table_pages, lengths, queries, query_stride, heads, cache->dtype, rule, out, out_dtype, lse, B, beam, n};
    if (const el_status st = check_attend(o, cache->kv_heads, cache->d_head, cache->page_size); st != EL_OK) return st;
    const AttendPlan p = plan_attend(*cache, heads, B, beam, n);
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return EL_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 15) return EL_ERR_INVALID_ARG;
    }
    const AttendArgs a = attend_args(o, page_view(*cache, table, table_stride, table_pages), cache->kv_heads, cache->d_head, lse, out, p, workspace);
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    launch_attend(a, p, cache->dtype, s);
    if (hipGetLastError() != hipSuccess) return EL_ERR_HIP;
    return p.spans ? launch_join(a, p, s) : EL_OK;
}
