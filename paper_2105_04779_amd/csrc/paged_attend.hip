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
// Work: the tiles of all sequences form one list, cut into as many equal spans as wavefronts (spans x units) fit the device at
// once.  A span that goes on to the next sequence closes a piece and starts another.  Every wavefront adds the lengths up by
// itself, so the cut follows them without the host knowing them.  Where sequences alone fill the device and are short, a
// wavefront takes one whole, and nothing is joined.
#include <cfloat>
#include <cmath>
#include <type_traits>
#include "mfma.h"
#include "paged.h"

namespace el {
namespace {

constexpr int kComputeUnits = 256, kDies = 8;                        // (a level-2 cache each)
constexpr int kLine = 128;           // bytes of a line of it
constexpr int kCrossing = 1;         // tiles that a span may be longer if it then starts with a sequence anew (find_span)
// Pieces of a sequence on average from which the join takes four wavefronts a row instead of one: one sequence of 16384 positions, one key head
// 20.7 us with four, 25.0 with one; 16 of 1000 to 4096, 32 rows on 8 key heads 50.8 / 47.0.
constexpr int64_t kManyPieces = 16;
// Tiles of a wavefront up to which a workgroup of several takes a whole sequence, without a second launch.  us on the device, cut and joined /
// whole: bf16, 16 heads of 64, 1 sequence of 613 9.9 / 9.5, 8 of 300 to 400 10.9 / 8.5, 16 of 400 to 800 17.0 / 13.3; 8 key heads of 128, 32 of
// 200 to 500 19.8 / 15.7, 1 of 500 (four tiles each) 11.0 / 12.6; fp32, 4 of 300 to 500 10.7 / 13.2.  Outside a graph the second launch and its
// scratch memory cost the host 5 us more than what the last two lose.  With eight tiles they lose 3 to 6 us.
// Of more sequences than find_span can start spans with, those that go on to the next cost more: 1000 of up to 300, one key head of 64,
// 30.2 / 14.6 (5 tiles each); 900 of up to 400, one of 128, 46.6 / 31.2 (13); 100 of up to 600 in fp32, two of 64, 21.9 / 16.8 (10); 70 of up to 2000, one
// of 64, 15.5 / 16.5 (16); 300 of up to 1000, two of 128, 45 / 58 (32).
constexpr int kFew = 4, kFewOfMany = 16;
// Positions that one wavefront may be left with where the sequences alone fill the device, so that nothing is joined: kShort, and as many for each
// time that they fill it as kRound bytes of keys have.  us, whole / cut: 16 heads of 64, 160 sequences of up to 700 59 / 62, of up to 1500 122 / 110;
// 600 of up to 2000 429 / 497; 8 heads of 128, 160 of up to 1000 86 / 74, 600 of up to 700 164 / 173.
constexpr int64_t kRound = 128 << 10;
constexpr int kShort = 2048;
// Sequences are never cut where there are more than kCutMost, whose lengths every wavefront would have to add up, and of more than kCutMax only
// longer ones: 8000 of up to 2500, one key head of 64, 447 us whole, 500 cut; 1500 of up to 8192, one of 128, 719 / 554.
constexpr int kCutMax = 1024, kCutMost = 1 << 14;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArgs {
    PageView c;
    const int32_t *lengths;
    const char *queries;
    int64_t query_stride;                    // bytes
    const float *slopes;
    // Scores stay as they leave the matrix unit; with a cap, a bias or a scale that is not positive (`shaped`) they are multiplied by `product` first
    // and kept in natural units.  `unit` > 0: powers of two in one of theirs, `natural`: e's.
    bool shaped;
    float product, softcap, unit, natural;
    int window, n, B, beam, heads, kv_heads, d;
    int group, R, row_blocks, rows;          // heads / kv_heads; query rows of a key head; blocks of them; rows of a block, at most
    bool near;                               // key heads that are neighbours in memory on one die
    int waves;                               // of a workgroup: a power of 2; more than one only where they share a whole sequence
    int spans;                               // spans that the tiles of all sequences are cut into, at most; 0: a span is a sequence
    void *out;
    int out_dtype;
    float *lse;
    int2 *pieces;                            // [B] first slot and number of slots of a sequence's pieces
    float *part_o;                           // [slot][unit][rows][d] weighted sums relative to part_ml's maximum
    float2 *part_ml;                         // [slot][unit][rows] (largest score, sum)
};

// Tiles [x, y) of a sequence of `len` positions.
__device__ __forceinline__ int length_of(const AttendArgs &a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.n) : a.n; }
__device__ __forceinline__ int2 tile_range(const AttendArgs &a, int len, int tile)
{
    const int first = a.window ? max(0, len - a.window) : 0;
    return int2{first / tile, (int)(((int64_t)len + tile - 1) / tile)};
}

// Where a span starts in the list of all sequences' tiles: sequence b, whose tiles are [before, before + ..) of the list.
struct Start { int b, before, at, end, T; bool aligned; };

// Sums over the lanes up to this one, on the vector ALU.
template <int CTRL, int ROWS> __device__ __forceinline__ int add_dpp(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int running_sum(int v)
{
    v = add_dpp<0x111, 0xf>(v);             // row_shr 1, 2, 4, 8: within 16 lanes
    v = add_dpp<0x112, 0xf>(v);
    v = add_dpp<0x114, 0xf>(v);
    v = add_dpp<0x118, 0xf>(v);
    v = add_dpp<0x142, 0xa>(v);             // the last lane of rows 0 and 2 to rows 1 and 3, then of lane 31 to the upper half
    return add_dpp<0x143, 0xc>(v);
}
__device__ __forceinline__ int sum_lanes(int v) { return __builtin_amdgcn_readlane(running_sum(v), 63); }

// Every wavefront adds the lengths up by itself: a lane those of a block of sequences, then the lanes theirs, and the block in which the span
// starts is looked through.  False: the list is shorter.
__device__ __forceinline__ bool find_span(const AttendArgs &a, int span, int tile, Start &s)
{
    const int lane = threadIdx.x, each = (a.B + 63) / 64;            // sequences of a block
    auto tiles_of = [&](int b, bool there) __attribute__((always_inline)) {          // (loaded in any case, so that many are on their way)
        const int2 r = tile_range(a, length_of(a, min(b, a.B - 1)), tile);
        return there ? r.y - r.x : 0;
    };
    int tiles = 0;
#pragma unroll 8
    for (int j = 0; j < each; ++j) tiles += tiles_of(lane * each + j, lane * each + j < a.B);
    int total = sum_lanes(tiles);
    s.T = max(1, (int)(((int64_t)total + a.spans - 1) / a.spans));
    s.aligned = false;
    if (each == 1) {
        // A span that goes on to another sequence goes the way through length, pages and first tile once more: where spans hardly longer
        // suffice that start with a sequence anew, they are taken (24 sequences with a window of 1024, d 256, 43 us; 51 with crossings).
        for (int T = s.T; T <= s.T + kCrossing && !s.aligned; ++T) {
            const int spans = sum_lanes((tiles + T - 1) / T);
            if (spans <= a.spans) { s.aligned = true; s.T = T; tiles = (tiles + T - 1) / T * T; total = spans * T; }
        }
    }
    if ((int64_t)span * s.T >= total) return false;
    s.at = span * s.T;
    s.end = (int)min((int64_t)s.at + s.T, (int64_t)total);
    s.before = 0;
    auto find = [&](int tiles) __attribute__((always_inline)) {      // the lane whose tiles hold the start, or -1: it lies behind them
        const int incl = running_sum(tiles);
        const unsigned long long past = __ballot(s.before + incl > s.at);
        const int first = past ? __ffsll((long long)past) - 1 : 63;
        s.before += __builtin_amdgcn_readlane(incl, first) - (past ? __builtin_amdgcn_readlane(tiles, first) : 0);
        return past ? first : -1;
    };
    s.b = find(tiles);
    if (each == 1) return true;
    const int b0 = s.b * each;
    for (int o = 0; o < each; o += 64) {
        const int i = find(tiles_of(b0 + o + lane, o + lane < each && b0 + o + lane < a.B));
        s.b = b0 + o + i;
        if (i >= 0) return true;
    }
    return false;
}

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

__device__ __forceinline__ float max_over_groups(float v)          // over the four lanes that hold one query row
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_groups(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

__device__ __forceinline__ void store4(void *out, int64_t at, int dtype, f4 v)
{
    if (dtype == EL_F32) *(f4 *)((float *)out + at) = v;
    else if (dtype == EL_F16) *(h4 *)((f16_t *)out + at) = __builtin_convertvector(v, h4);
    else *(u2 *)((uint16_t *)out + at) = u2{__builtin_bit_cast(unsigned, __builtin_convertvector(f2{v[0], v[1]}, b2)),
                                            __builtin_bit_cast(unsigned, __builtin_convertvector(f2{v[2], v[3]}, b2))};
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

// Joins the pieces of a sequence that was cut: PER wavefronts a (sequence, query row, head), 4 / PER of those a workgroup.  Bound by
// latency, so the first weighted sums are requested together with the statistics.
template <int PER>
__global__ void __launch_bounds__(256) k_attend_join(const AttendArgs a, int tile)
{
    __shared__ float red[PER == 1 ? 1 : 8];
    __shared__ f4 sums[PER == 1 ? 1 : 256];
    constexpr int LANES = 64 * PER, AHEAD = 4;
    const int tid = threadIdx.x % LANES, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * (4 / PER) + (PER == 1 ? w : 0);
    if (row >= (int64_t)a.B * a.beam * a.heads) return;
    const int b = (int)(row / (a.beam * a.heads)), x = (int)(row - (int64_t)b * (a.beam * a.heads));
    const int2 pc = a.pieces[b];                                     // (not written for a sequence without a tile)
    const int2 range = tile_range(a, length_of(a, b), tile);
    if (range.y == range.x) {
        if (tid < a.d / 4) store4(a.out, row * a.d + 4 * tid, a.out_dtype, f4{0.f, 0.f, 0.f, 0.f});
        if (tid == 0 && a.lse) a.lse[row] = -INFINITY;
        return;
    }
    if (pc.y < 2) return;
    const int j = x / a.heads, head = x - j * a.heads, kvh = head / a.group, r = j * a.group + head % a.group;
    const int units = a.kv_heads * a.row_blocks, unit = r / a.rows * a.kv_heads + kvh, rb = r % a.rows;
    const int64_t first = ((int64_t)pc.x * units + unit) * a.rows + rb, step = (int64_t)units * a.rows;
    const float2 *const ml = a.part_ml + first;
    const int d4 = a.d / 4, groups = LANES / d4, grp = tid / d4, col = tid - grp * d4;
    const float *const po = a.part_o + first * a.d + 4 * col;
    const int begin = grp < groups ? grp : pc.y;
    f4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        ahead[i] = f4{0.f, 0.f, 0.f, 0.f};
        if (begin + i * groups < pc.y) ahead[i] = *(const f4 *)(po + (begin + i * groups) * step * a.d);
    }
    float M = -INFINITY;
    for (int s = tid; s < pc.y; s += LANES) M = fmaxf(M, ml[s * step].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    if constexpr (PER > 1) {
        if (lane == 0) red[w] = M;
        __syncthreads();
        M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
    const float ref = M == -INFINITY ? 0.f : M;
    // (a piece without a position: sum 0.  A NaN score leaves its maximum at -inf and its sum at NaN, which stays)
    auto weight = [&](float m) __attribute__((always_inline)) { return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - ref) * a.unit); };
    float L = 0.f;
    for (int s = tid; s < pc.y; s += LANES) {
        const float2 v = ml[s * step];
        L += weight(v.x) * v.y;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o, 64);
    if constexpr (PER > 1) {
        if (lane == 0) red[4 + w] = L;
        __syncthreads();
        L = (red[4] + red[5]) + (red[6] + red[7]);
    }
    const bool empty = M == -INFINITY && !(L != L);
    if (tid == 0 && a.lse) a.lse[row] = empty ? -INFINITY : fmaf(M, a.natural, __builtin_amdgcn_logf(L) * kLn2);
    f4 o{0.f, 0.f, 0.f, 0.f};
    auto add = [&](const f4 &v, float f) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f * v[e];
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (begin + i * groups < pc.y) add(ahead[i], weight(ml[(begin + i * groups) * step].x));
#pragma unroll 8
    for (int s = begin + AHEAD * groups; s < pc.y; s += groups) add(*(const f4 *)(po + s * step * a.d), weight(ml[s * step].x));
    if constexpr (PER > 1) {
        sums[tid] = o;
        __syncthreads();
        if (tid < d4)
            for (int k = 1; k < groups; ++k) add(sums[k * d4 + tid], 1.f);
    } else {
        for (int k = 1; k < groups; ++k) {
            f4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __shfl(o[e], min(lane + k * d4, 63), 64);
            if (lane < d4) add(v, 1.f);
        }
    }
    if (tid < d4) {
        const float inv = 1.f / L;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = empty ? 0.f : o[e] * inv;
        store4(a.out, row * a.d + 4 * tid, a.out_dtype, o);
    }
}

// What a call is launched with: host arithmetic.
struct AttendPlan { int padded, row_groups, row_blocks, rows, tile, waves, spans, grid, lds; bool near; size_t pieces_bytes, ml_bytes, workspace; };

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
    AttendPlan p;
    const int R = beam * (heads / c.kv_heads);
    p.padded = c.d_head <= 64 ? 64 : c.d_head <= 128 ? 128 : 256;
    // Two groups of rows share a tile's operand reads; in fp32 beyond 128 columns their registers do not suffice.  (Four, for more than 32
    // rows, gain nothing sure: 16 sequences of 1000 to 4096, 8 key heads of 128, 64 rows 75 us with two blocks of two / 70 with one of four,
    // 16 key heads of 64 51 / 55.)
    p.row_groups = R <= 16 || (c.dtype == EL_F32 && p.padded == 256) ? 1 : 2;
    p.row_blocks = (R + 16 * p.row_groups - 1) / (16 * p.row_groups);
    p.rows = R < 16 * p.row_groups ? R : 16 * p.row_groups;
    const int64_t units = (int64_t)c.kv_heads * p.row_blocks;
    int slots = 0, most = 1, lds = 0;
    with_form(c.dtype, p.padded, p.row_groups, [&](auto f) { p.tile = f.TP; slots = kComputeUnits * f.PER_CU; most = f.WAVES; lds = f.LDS; });
    const int64_t tiles = ((int64_t)n + p.tile - 1) / p.tile, all = B * tiles;
    // spans: one round of wavefronts; where the units are so many that one round would leave much of the device idle, four
    const int64_t target = units <= slots / 8 ? slots / units : (4 * (int64_t)slots + units - 1) / units;
    p.waves = 1;
    while (p.waves < most && 2 * p.waves * B * units <= slots && 2 * p.waves <= tiles) p.waves *= 2;
    // whole sequences: where they alone fill the device and none is long, where the lengths would take long to add up, and where a few
    // tiles are all that a wavefront gets
    const int64_t key_bytes = p.padded * (int64_t)dtype_size(c.dtype);
    const bool few = tiles <= (int64_t)(B > 64 ? kFewOfMany : kFew) * p.waves;
    const bool fill = B * units >= slots && n <= kShort && n * key_bytes * slots <= kRound * B * units;
    const bool whole = few || fill || (B > kCutMax && n <= 2 * kShort) || B > kCutMost || all > 1 << 30;
    if (!whole) p.waves = 1;
    p.spans = whole ? 0 : (int)(target < all ? target : all);
    p.grid = (int)((whole ? B : p.spans) * units);
    // Heads that share lines are read by one die, or each of the two fetches them: 500 sequences of 500 to 700, 16 heads of 32, 159 us, 233 apart;
    // 16 of 1000 to 3000, 5 rows on each of 20 heads of 40, 41 / 54; 100 of 100 to 2500, 16 heads of 80, 155 / 182.  So are heads of one line each where
    // wavefronts take whole sequences: 500 of 512 to 1024, 16 heads of 64, 265 / 299.  In spans, with few heads and at longer rows apart is better by up to 5 %
    // (150 of up to 2500 167, 174 near; 600 of 500 to 700, 4 heads, 81 / 83; 300 of 100 to 800, 8 heads of 128, 115 / 118).
    const int64_t head_bytes = c.head_stride * (int64_t)dtype_size(c.dtype);
    p.near = head_bytes % kLine != 0 || (head_bytes == kLine && whole && p.waves == 1 && units >= kDies);
    p.lds = p.waves * lds;
    p.pieces_bytes = p.ml_bytes = p.workspace = 0;
    if (p.spans) {
        const size_t rows = ((size_t)p.spans + B) * units * p.rows;
        p.pieces_bytes = align_up((size_t)B * sizeof(int2), 256);
        p.ml_bytes = align_up(rows * sizeof(float2), 256);
        p.workspace = p.pieces_bytes + p.ml_bytes + rows * c.d_head * sizeof(float);
    }
    return p;
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

bool finite_non_negative(float x) { return x >= 0.f && x < INFINITY; }

constexpr int64_t kMaxRows = (int64_t)1 << 23;                       // B x beam x heads: a launch has fewer than 2^32 threads

bool valid_sizes(const el_attn_pages *c, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    return heads >= 1 && B >= 1 && beam >= 1 && n >= 1 && heads % c->kv_heads == 0 && (int64_t)B * beam <= kMaxRows && (int64_t)B * beam * heads <= kMaxRows;
}

} // namespace
} // namespace el

extern "C" size_t el_attn_paged_workspace_bytes(const el_attn_pages *cache, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    if (el::check_pages(cache) != EL_OK || !el::valid_sizes(cache, heads, B, beam, n)) return 0;
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
    if (const el_status st = check_table(table, table_stride, table_pages, B); st != EL_OK) return st;
    if (!queries || !rule || !out || !valid_sizes(cache, heads, B, beam, n)) return EL_ERR_INVALID_ARG;
    if (out_dtype != EL_F32 && out_dtype != cache->dtype) return EL_ERR_UNSUPPORTED;
    if (n > (int64_t)table_pages * cache->page_size) return EL_ERR_INVALID_ARG;
    if (!finite_non_negative(rule->softcap) || rule->window < 0) return EL_ERR_INVALID_ARG;
    if (!(fabsf(rule->softcap > 0.f ? rule->scale / rule->softcap : rule->scale * kLog2e) < INFINITY)) return EL_ERR_INVALID_ARG;
    const int64_t es = (int64_t)dtype_size(cache->dtype), row = (int64_t)heads * cache->d_head, rows = (int64_t)B * beam;
    if (((uintptr_t)lengths | (uintptr_t)lse | (uintptr_t)rule->slopes) & 3 || ((uintptr_t)queries | (uintptr_t)out) & 15) return EL_ERR_INVALID_ARG;
    if (query_stride > ((int64_t)1 << 44) || query_stride * es % 16 != 0 || (rows > 1 && query_stride < row) || out_of_reach(rows, query_stride * es)) return EL_ERR_INVALID_ARG;
    // (several wavefronts read a query row, and one that is done writes its part of the output)
    const uintptr_t q0 = (uintptr_t)queries, q1 = q0 + (uintptr_t)((rows > 1 ? (rows - 1) * query_stride : 0) + row) * es;
    const uintptr_t o0 = (uintptr_t)out, o1 = o0 + (uintptr_t)(rows * row) * dtype_size(out_dtype);
    if (q0 < o1 && o0 < q1) return EL_ERR_INVALID_ARG;
    const AttendPlan p = plan_attend(*cache, heads, B, beam, n);
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return EL_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 15) return EL_ERR_INVALID_ARG;
    }
    AttendArgs a{};
    a.c = page_view(*cache, table, table_stride, table_pages);
    a.lengths = lengths;
    a.queries = (const char *)queries; a.query_stride = query_stride * es;
    a.slopes = rule->slopes; a.softcap = rule->softcap; a.window = rule->window;
    a.shaped = rule->softcap > 0.f || rule->slopes || !(rule->scale >= FLT_MIN);
    a.product = rule->softcap > 0.f ? rule->scale / rule->softcap : rule->scale;
    a.unit = a.shaped ? kLog2e : rule->scale * kLog2e;
    a.natural = a.shaped ? 1.f : rule->scale;
    a.n = n; a.B = B; a.beam = beam; a.heads = heads; a.kv_heads = cache->kv_heads; a.d = cache->d_head;
    a.group = heads / cache->kv_heads; a.R = beam * a.group; a.row_blocks = p.row_blocks; a.rows = p.rows;
    a.near = p.near; a.waves = p.waves; a.spans = p.spans;
    a.out = out; a.out_dtype = out_dtype; a.lse = lse;
    if (p.workspace) {
        a.pieces = (int2 *)workspace;
        a.part_ml = (float2 *)((char *)workspace + p.pieces_bytes);
        a.part_o = (float *)((char *)workspace + p.pieces_bytes + p.ml_bytes);
    }
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    launch_attend(a, p, cache->dtype, s);
    if (hipGetLastError() != hipSuccess) return EL_ERR_HIP;
    if (p.spans) {
        // four wavefronts a row where sequences are cut into many pieces
        const int64_t all = rows * heads;
        if (p.spans > kManyPieces * B) hipLaunchKernelGGL(k_attend_join<4>, dim3((unsigned)all), dim3(256), 0, s, a, p.tile);
        else hipLaunchKernelGGL(k_attend_join<1>, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, p.tile);
        if (hipGetLastError() != hipSuccess) return EL_ERR_HIP;
    }
    return EL_OK;
}
