// What the attentions over pages share: the cut of all sequences' tiles into spans, the join of a sequence's pieces, and their checks.
//
// The tiles of all sequences form one list, cut into as many equal spans as wavefronts (spans x units) fit the device at once.  A span that
// goes on to the next sequence closes a piece and starts another.  Every wavefront adds the lengths up by itself, so the cut follows them
// without the host knowing them.  Where sequences alone fill the device and are short, a wavefront takes one whole, and nothing is joined.
#pragma once
#include <cfloat>
#include <cmath>
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

// What a wavefront of an attention is built for: d_head padded, query rows in groups of 16, positions of a tile; wavefronts that a compute unit
// holds, and that share a sequence, at most; bytes of LDS of each.
struct SpanForm { int padded, row_groups, tile, per_cu, most, lds; };

// What a call is launched with: host arithmetic.
struct AttendPlan { int padded, row_groups, row_blocks, rows, tile, waves, spans, grid, lds; bool near; size_t pieces_bytes, ml_bytes, workspace; };

// R: query rows of a key head; key_bytes: of a padded key; head_bytes: from a key head to the next.
inline AttendPlan plan_spans(const SpanForm &form, int R, int kv_heads, int d_head, int64_t key_bytes, int64_t head_bytes, int B, int n)
{
    AttendPlan p;
    p.padded = form.padded; p.row_groups = form.row_groups; p.tile = form.tile;
    p.row_blocks = (R + 16 * p.row_groups - 1) / (16 * p.row_groups);
    p.rows = R < 16 * p.row_groups ? R : 16 * p.row_groups;
    const int64_t units = (int64_t)kv_heads * p.row_blocks;
    const int slots = kComputeUnits * form.per_cu;
    const int64_t tiles = ((int64_t)n + p.tile - 1) / p.tile, all = B * tiles;
    // spans: one round of wavefronts; where the units are so many that one round would leave much of the device idle, four
    const int64_t target = units <= slots / 8 ? slots / units : (4 * (int64_t)slots + units - 1) / units;
    p.waves = 1;
    while (p.waves < form.most && 2 * p.waves * B * units <= slots && 2 * p.waves <= tiles) p.waves *= 2;
    // whole sequences: where they alone fill the device and none is long, where the lengths would take long to add up, and where a few
    // tiles are all that a wavefront gets
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
    p.near = head_bytes % kLine != 0 || (head_bytes == kLine && whole && p.waves == 1 && units >= kDies);
    p.lds = p.waves * form.lds;
    p.pieces_bytes = p.ml_bytes = p.workspace = 0;
    if (p.spans) {
        const size_t rows = ((size_t)p.spans + B) * units * p.rows;
        p.pieces_bytes = align_up((size_t)B * sizeof(int2), 256);
        p.ml_bytes = align_up(rows * sizeof(float2), 256);
        p.workspace = p.pieces_bytes + p.ml_bytes + rows * d_head * sizeof(float);
    }
    return p;
}

inline bool finite_non_negative(float x) { return x >= 0.f && x < INFINITY; }

constexpr int64_t kMaxRows = (int64_t)1 << 23;                       // B x beam x heads: a launch has fewer than 2^32 threads

inline bool valid_sizes(int32_t kv_heads, int32_t heads, int32_t B, int32_t beam, int32_t n)
{
    return heads >= 1 && B >= 1 && beam >= 1 && n >= 1 && heads % kv_heads == 0 && (int64_t)B * beam <= kMaxRows && (int64_t)B * beam * heads <= kMaxRows;
}

// What a call of an attention is given beside the cache.
struct AttendOperands {
    const int32_t *table; int64_t table_stride; int32_t table_pages;
    const int32_t *lengths;
    const void *queries; int64_t query_stride; int32_t heads; int32_t dtype;
    const el_attn_score_rule *rule;
    const void *out; int32_t out_dtype; const float *lse;
    int32_t B, beam, n;
};

// Host: the checks of an attention's operands, for a cache that has been found to be one.
inline el_status check_attend(const AttendOperands &o, int32_t kv_heads, int32_t d_head, int32_t page_size)
{
    if (const el_status st = check_table(o.table, o.table_stride, o.table_pages, o.B); st != EL_OK) return st;
    if (!o.queries || !o.rule || !o.out || !valid_sizes(kv_heads, o.heads, o.B, o.beam, o.n)) return EL_ERR_INVALID_ARG;
    if (o.out_dtype != EL_F32 && o.out_dtype != o.dtype) return EL_ERR_UNSUPPORTED;
    if (o.n > (int64_t)o.table_pages * page_size) return EL_ERR_INVALID_ARG;
    const el_attn_score_rule &rule = *o.rule;
    if (!finite_non_negative(rule.softcap) || rule.window < 0) return EL_ERR_INVALID_ARG;
    if (!(fabsf(rule.softcap > 0.f ? rule.scale / rule.softcap : rule.scale * kLog2e) < INFINITY)) return EL_ERR_INVALID_ARG;
    const int64_t es = (int64_t)dtype_size(o.dtype), row = (int64_t)o.heads * d_head, rows = (int64_t)o.B * o.beam;
    if (((uintptr_t)o.lengths | (uintptr_t)o.lse | (uintptr_t)rule.slopes) & 3 || ((uintptr_t)o.queries | (uintptr_t)o.out) & 15) return EL_ERR_INVALID_ARG;
    if (o.query_stride > ((int64_t)1 << 44) || o.query_stride * es % 16 != 0 || (rows > 1 && o.query_stride < row) || out_of_reach(rows, o.query_stride * es)) return EL_ERR_INVALID_ARG;
    // (several wavefronts read a query row, and one that is done writes its part of the output)
    const uintptr_t q0 = (uintptr_t)o.queries, q1 = q0 + (uintptr_t)((rows > 1 ? (rows - 1) * o.query_stride : 0) + row) * es;
    const uintptr_t o0 = (uintptr_t)o.out, o1 = o0 + (uintptr_t)(rows * row) * dtype_size(o.out_dtype);
    if (q0 < o1 && o0 < q1) return EL_ERR_INVALID_ARG;
    return EL_OK;
}

// The arguments of a launch, for operands that have passed; pieces and partial results in the workspace.
inline AttendArgs attend_args(const AttendOperands &o, const PageView &view, int32_t kv_heads, int32_t d_head, float *lse, void *out,
                              const AttendPlan &p, void *workspace)
{
    const el_attn_score_rule &rule = *o.rule;
    AttendArgs a{};
    a.c = view;
    a.lengths = o.lengths;
    a.queries = (const char *)o.queries; a.query_stride = o.query_stride * (int64_t)dtype_size(o.dtype);
    a.slopes = rule.slopes; a.softcap = rule.softcap; a.window = rule.window;
    a.shaped = rule.softcap > 0.f || rule.slopes || !(rule.scale >= FLT_MIN);
    a.product = rule.softcap > 0.f ? rule.scale / rule.softcap : rule.scale;
    a.unit = a.shaped ? kLog2e : rule.scale * kLog2e;
    a.natural = a.shaped ? 1.f : rule.scale;
    a.n = o.n; a.B = o.B; a.beam = o.beam; a.heads = o.heads; a.kv_heads = kv_heads; a.d = d_head;
    a.group = o.heads / kv_heads; a.R = o.beam * a.group; a.row_blocks = p.row_blocks; a.rows = p.rows;
    a.near = p.near; a.waves = p.waves; a.spans = p.spans;
    a.out = out; a.out_dtype = o.out_dtype; a.lse = lse;
    if (p.workspace) {
        a.pieces = (int2 *)workspace;
        a.part_ml = (float2 *)((char *)workspace + p.pieces_bytes);
        a.part_o = (float *)((char *)workspace + p.pieces_bytes + p.ml_bytes);
    }
    return a;
}

// The second launch of a call whose sequences are cut.
inline el_status launch_join(const AttendArgs &a, const AttendPlan &p, hipStream_t s)
{
    // four wavefronts a row where sequences are cut into many pieces
    const int64_t all = (int64_t)a.B * a.beam * a.heads;
    if (p.spans > kManyPieces * a.B) hipLaunchKernelGGL(k_attend_join<4>, dim3((unsigned)all), dim3(256), 0, s, a, p.tile);
    else hipLaunchKernelGGL(k_attend_join<1>, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, p.tile);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}

} // namespace
} // namespace el
