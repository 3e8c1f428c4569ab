// The table of the next step: who goes on from whom, pages for new positions, copies of shared pages that are written, a slot for every new position.
//
// Pages in use are those that the new sequences name, so nothing is kept between calls.  Bound by latency at the sizes of a serving batch: one launch of one
// workgroup where little is to be done (k_plan_small), else four: marks cleared; rows copied and their pages marked; the unmarked pages of each chunk listed, and
// every sequence's need added up; entries, slots.  512 requests of up to 8192 positions on 1.5 times the pages they need: 2.5 + 8.4 + 5.8 + 6.2 us.
//
// A mark is the largest of the keys (positions of the page in use, written?, lowest sequence first) of those that name it: a page is its writer's to keep if the
// mark is the writer's own key.  Where a write changes more than the positions written (a cache in 8 bits), it is the number of entries that name the page, and a page is
// its writer's to keep if that is 1.  Maxima and whole-number sums: the result does not depend on the order in which anything runs.
#include "el_internal.h"

namespace el {
namespace {

constexpr int kChunk = 4096;             // pages of a chunk
constexpr int kLanes = 256;
constexpr int kMaxPages = 1 << 24, kMaxSequences = 1 << 20;
constexpr int kMostChunks = kMaxPages / kChunk;

typedef unsigned long long Mark;

struct PlanArgs {
    const int32_t *table; int64_t table_stride;
    const int32_t *lengths, *parents, *counts;
    const uint8_t *reserved;
    int columns, B_old, pages, page_size, B, T, chunks;
    bool exclusive;                      // a page that is written is named once
    int32_t *new_table, *new_lengths, *granted, *copies, *free_pages;
    int64_t *slots;
    Mark *marks;                         // [pages]
    int32_t *free_list, *free_count;     // [chunk][kChunk] its unmarked pages in ascending order; [chunk]
    int64_t *before, *block_need;        // [B] pages needed by those before in the block of kLanes, times 2, plus 1 where a page is replaced; [block]
    int32_t *need;                       // [B]
};

// What sequence b goes on from and asks for.
struct Ask { const int32_t *row; int had, count, held, held_then; };
__device__ __forceinline__ Ask ask(const PlanArgs &a, int b)
{
    const int p = a.parents ? a.parents[b] : b;
    const bool there = p >= 0 && p < a.B_old;
    Ask s;
    s.row = a.table + (there ? p : 0) * a.table_stride;
    const int most = a.columns * a.page_size;                        // (below 2^31)
    s.had = there ? min(max(a.lengths[p], 0), most) : 0;
    s.count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
    if (s.count > most - s.had) s.count = 0;                         // more than the columns hold
    s.held = (int)(((int64_t)s.had + a.page_size - 1) / a.page_size);
    s.held_then = (int)(((int64_t)s.had + s.count + a.page_size - 1) / a.page_size);
    return s;
}
__device__ __forceinline__ int entry(const PlanArgs &a, const Ask &s, int j)
{
    const int e = j < s.held ? s.row[j] : -1;
    return e >= 0 && e < a.pages ? e : -1;
}
__device__ __forceinline__ bool writes_last(const PlanArgs &a, const Ask &s) { return s.count > 0 && s.had % a.page_size != 0; }
__device__ __forceinline__ Mark key_of(const PlanArgs &a, const Ask &s, int j, int b)
{
    const int extent = min(a.page_size, s.had - j * a.page_size);
    return (Mark)extent << 32 | (j == s.held - 1 && writes_last(a, s) ? (1u << 31) + (unsigned)(kMaxSequences - b) : 0u);
}
__device__ __forceinline__ void mark(const PlanArgs &a, Mark *at, const Ask &s, int j, int b)
{
    if (a.exclusive) atomicAdd(at, (Mark)1);
    else atomicMax(at, key_of(a, s, j, b));
}
// Is a page with this mark, the last of s, the writer's to keep?
__device__ __forceinline__ bool keeps(const PlanArgs &a, Mark m, const Ask &s, int b) { return m == (a.exclusive ? (Mark)1 : key_of(a, s, s.held - 1, b)); }

__global__ void __launch_bounds__(256) k_plan_clear(Mark *marks, int pages)
{
    for (int i = blockIdx.x * 256 + threadIdx.x; i < pages; i += gridDim.x * 256) marks[i] = 0;
}

// Grid: (parts of a row, B).
__global__ void __launch_bounds__(kLanes) k_plan_mark(const PlanArgs a)
{
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        const Ask s = ask(a, b);
        for (int j = blockIdx.x * kLanes + threadIdx.x; j < a.columns; j += gridDim.x * kLanes) {
            const int e = entry(a, s, j);
            a.new_table[(int64_t)b * a.columns + j] = e;
            if (e >= 0) mark(a, &a.marks[e], s, j, b);
        }
    }
}

// Sum over the lanes of a workgroup up to and without this one's; `total`: of all.
template <int LANES = kLanes>
__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t &total)
{
    __shared__ int64_t part[LANES / 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t up = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int64_t x = __shfl_up(up, o, 64); if (lane >= o) up += x; }
    __syncthreads();
    if (lane == 63) part[w] = up;
    __syncthreads();
    int64_t first = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) { if (i < w) first += part[i]; total += part[i]; }
    return first + up - v;
}

// Grid: chunks of pages, then blocks of sequences.
__global__ void __launch_bounds__(kLanes) k_plan_count(const PlanArgs a)
{
    int64_t total;
    if ((int)blockIdx.x < a.chunks) {
        const int first = blockIdx.x * kChunk + threadIdx.x * (kChunk / kLanes);
        unsigned free = 0;
#pragma unroll
        for (int i = 0; i < kChunk / kLanes; ++i) {
            const int p = first + i;
            if (p < a.pages && a.marks[p] == 0 && !(a.reserved && a.reserved[p])) free |= 1u << i;
        }
        int at = (int)sum_before(__popc(free), total);
        for (; free; free &= free - 1) a.free_list[(int64_t)blockIdx.x * kChunk + at++] = first + __ffs((int)free) - 1;
        if (threadIdx.x == 0) a.free_count[blockIdx.x] = (int)total;
        return;
    }
    const int block = blockIdx.x - a.chunks, b = block * kLanes + threadIdx.x;
    int need = 0;
    bool replaced = false;
    if (b < a.B) {
        const Ask s = ask(a, b);
        if (writes_last(a, s)) {
            const int e = entry(a, s, s.held - 1);
            replaced = e < 0 || (a.reserved && a.reserved[e]) || !keeps(a, a.marks[e], s, b);
        }
        if (s.count > 0) need = s.held_then - s.held + replaced;
    }
    const int64_t before = sum_before(need, total);
    if (b < a.B) { a.before[b] = 2 * before + replaced; a.need[b] = need; }
    if (threadIdx.x == 0) a.block_need[block] = total;
}

// Sum of values[0 .. n) over a workgroup.
template <typename T>
__device__ __forceinline__ int64_t sum_of(const T *values, int n)
{
    int64_t v = 0, total;
    for (int i = threadIdx.x; i < n; i += kLanes) v += values[i];
    (void)sum_before(v, total);
    return total;
}

// Grid: a sequence a workgroup, and one more for the pages left.
__global__ void __launch_bounds__(kLanes) k_plan_assign(const PlanArgs a)
{
    __shared__ int64_t chunk_before[kMostChunks + 1];                // free pages before each chunk, and all
    {
        const int each = (a.chunks + kLanes - 1) / kLanes, first = threadIdx.x * each;
        int64_t mine = 0, total;
        for (int i = first; i < min(first + each, a.chunks); ++i) mine += a.free_count[i];
        int64_t at = sum_before(mine, total);
        for (int i = first; i < min(first + each, a.chunks); ++i) { chunk_before[i] = at; at += a.free_count[i]; }
        if (threadIdx.x == 0) chunk_before[a.chunks] = total;
    }
    __syncthreads();
    const int64_t available = chunk_before[a.chunks];
    if ((int)blockIdx.x == a.B) {
        // all that is granted is a beginning of what is needed: the largest sum that the free pages suffice for
        const int blocks = (a.B + kLanes - 1) / kLanes;
        int64_t first = 0, most = 0;
        for (int k = 0; k < blocks; ++k) {
            const int b = k * kLanes + threadIdx.x;
            if (b < a.B) { const int64_t upto = first + a.before[b] / 2 + a.need[b]; if (upto <= available && upto > most) most = upto; }
            first += a.block_need[k];
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { const int64_t x = __shfl_xor(most, o, 64); if (x > most) most = x; }
        __shared__ int64_t part[kLanes / 64];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < kLanes / 64; ++i) if (part[i] > most) most = part[i];
            a.free_pages[0] = (int)(available - most);
        }
        return;
    }
    const int b = blockIdx.x;
    const Ask s = ask(a, b);
    const int need = a.need[b];
    const bool replaced = a.before[b] & 1;
    const int64_t before = sum_of(a.block_need, b / kLanes) + a.before[b] / 2;
    const bool grant = s.count > 0 && (need == 0 || before + need <= available);
    const int granted = grant ? s.count : 0;
    auto nth_free = [&](int64_t i) {                                 // the i-th free page
        int lo = 0, hi = a.chunks - 1;
        while (lo < hi) { const int mid = (lo + hi + 1) / 2; if (chunk_before[mid] <= i) lo = mid; else hi = mid - 1; }
        return a.free_list[(int64_t)lo * kChunk + (i - chunk_before[lo])];
    };
    auto page_of = [&](int j) {                                      // of column j, below those held then
        if (grant && replaced && j == s.held - 1) return nth_free(before);
        if (j < s.held) return entry(a, s, j);
        return nth_free(before + replaced + j - s.held);
    };
    if (grant) {
        const int from = s.held - (replaced ? 1 : 0);
        for (int j = from + threadIdx.x; j < s.held_then; j += kLanes) a.new_table[(int64_t)b * a.columns + j] = page_of(j);
    }
    if (a.slots)
        for (int i = threadIdx.x; i < a.T; i += kLanes) {
            int64_t slot = -1;
            if (i < granted) {
                const int at = s.had + i, j = at / a.page_size, page = page_of(j);
                slot = (int64_t)page * a.page_size + (at - j * a.page_size);
            }
            a.slots[(int64_t)b * a.T + i] = slot;
        }
    if (threadIdx.x == 0) {
        a.new_lengths[b] = s.had + granted;
        a.granted[b] = granted;
        const int src = grant && replaced ? entry(a, s, s.held - 1) : -1;
        a.copies[b] = src;
        a.copies[a.B + b] = src >= 0 ? nth_free(before) : -1;
        a.copies[2 * a.B + b] = src >= 0 ? s.had % a.page_size : 0;
    }
}

// All of it by one workgroup, marks and free pages in LDS: pools of kSmallPages at most, where few entries and slots are to be gone through.  us on the device, four
// launches / one: 32 sequences of 10 pages 15.2 / 8.8, 128 of 32 15.3 / 12.3, 64 of 128 16.3 / 15.3 (8256 entries and slots), 256 of 32 16.3 / 16.7, 64 of 119 and 128
// new positions each 16.3 / 22.3.  Outside a graph three launches less save the host as much again.
constexpr int kSmallPages = 8192, kSmallLanes = 1024;
constexpr int64_t kSmallWork = 1 << 13;
__global__ void __launch_bounds__(kSmallLanes) k_plan_small(const PlanArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char shared[];
    Mark *const marks = (Mark *)shared;                              // [pages]
    int *const list = (int *)(marks + a.pages);                      // [pages] free pages, ascending
    __shared__ int first_page[kSmallLanes];                          // of a sequence, of the free ones: its first; -1: nothing granted
    __shared__ bool replaces[kSmallLanes];
    const int tid = threadIdx.x;
    for (int i = tid; i < a.pages; i += kSmallLanes) marks[i] = 0;
    __syncthreads();
    for (int i = tid; i < a.B * a.columns; i += kSmallLanes) {
        const int b = i / a.columns, j = i - b * a.columns;
        const Ask s = ask(a, b);
        const int e = entry(a, s, j);
        a.new_table[i] = e;
        if (e >= 0) mark(a, &marks[e], s, j, b);
    }
    __syncthreads();
    int64_t available, all;
    {
        constexpr int EACH = kSmallPages / kSmallLanes;
        unsigned free = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = tid * EACH + i;
            if (p < a.pages && marks[p] == 0 && !(a.reserved && a.reserved[p])) free |= 1u << i;
        }
        int at = (int)sum_before<kSmallLanes>(__popc(free), available);
        for (; free; free &= free - 1) list[at++] = tid * EACH + __ffs((int)free) - 1;
    }
    // a sequence a lane
    Ask s{};
    int need = 0, last = -1;
    bool replaced = false;
    if (tid < a.B) {
        s = ask(a, tid);
        if (writes_last(a, s)) {
            last = entry(a, s, s.held - 1);
            replaced = last < 0 || (a.reserved && a.reserved[last]) || !keeps(a, marks[last], s, tid);
        }
        if (s.count > 0) need = s.held_then - s.held + replaced;
    }
    const int64_t before = sum_before<kSmallLanes>(need, all);       // (and the list is there for all)
    const bool grant = s.count > 0 && (need == 0 || before + need <= available);
    if (tid < a.B) {
        const int at = (int)before, granted = grant ? s.count : 0;
        first_page[tid] = grant ? at : -1;
        replaces[tid] = replaced;
        if (grant) {
            if (replaced) a.new_table[tid * a.columns + s.held - 1] = list[at];
            for (int j = s.held; j < s.held_then; ++j) a.new_table[tid * a.columns + j] = list[at + replaced + j - s.held];
        }
        a.new_lengths[tid] = s.had + granted;
        a.granted[tid] = granted;
        const int src = grant && replaced ? last : -1;
        a.copies[tid] = src;
        a.copies[a.B + tid] = src >= 0 ? list[at] : -1;
        a.copies[2 * a.B + tid] = src >= 0 ? s.had % a.page_size : 0;
    }
    // all that is granted is a beginning of what is needed
    int64_t granted_pages;
    (void)sum_before<kSmallLanes>(before + need <= available ? need : 0, granted_pages);
    if (tid == 0) a.free_pages[0] = (int)(available - granted_pages);
    __syncthreads();
    if (a.slots)
        for (int i = tid; i < a.B * a.T; i += kSmallLanes) {
            const int b = i / a.T, t = i - b * a.T, at = first_page[b];
            int64_t slot = -1;
            if (at >= 0) {
                const Ask x = ask(a, b);
                if (t < x.count) {
                    const int position = x.had + t, j = position / a.page_size;
                    const bool anew = replaces[b];
                    const int page = j < x.held - (anew ? 1 : 0) ? entry(a, x, j) : list[at + j - (x.held - (anew ? 1 : 0))];
                    slot = (int64_t)page * a.page_size + (position - j * a.page_size);
                }
            }
            a.slots[i] = slot;
        }
}

struct PlanSpace { size_t marks, list, count, before, block_need, need, total; int chunks; };
PlanSpace plan_space(int32_t B, int32_t pages)
{
    PlanSpace p;
    p.chunks = (pages + kChunk - 1) / kChunk;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
    p.marks = take((size_t)pages * sizeof(Mark));
    p.list = take((size_t)p.chunks * kChunk * sizeof(int32_t));
    p.count = take((size_t)p.chunks * sizeof(int32_t));
    p.before = take((size_t)B * sizeof(int64_t));
    p.block_need = take((size_t)(B + kLanes - 1) / kLanes * sizeof(int64_t));
    p.need = take((size_t)B * sizeof(int32_t));
    p.total = at;
    return p;
}

// The checks and launches of both calls.
el_status plan(bool exclusive, const int32_t *table, int64_t table_stride, int32_t columns, const int32_t *lengths, int32_t B_old,
               const int32_t *parents, const int32_t *counts, const uint8_t *reserved, int32_t pages, int32_t page_size,
               int32_t B, int32_t T, int32_t *new_table, int32_t *new_lengths, int32_t *granted, int64_t *slots,
               int32_t *copies, int32_t *free_pages, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!table || !lengths || !new_table || !new_lengths || !granted || !copies || !free_pages) return EL_ERR_INVALID_ARG;
    if (columns < 1 || columns > 1 << 24 || B_old < 1 || B_old > kMaxSequences || B < 1 || B > kMaxSequences || T < 1 || T > 1 << 23 ||
        pages < 1 || pages > kMaxPages || page_size < 1 || (int64_t)columns * page_size > INT32_MAX || (int64_t)B * columns > ((int64_t)1 << 31)) return EL_ERR_INVALID_ARG;
    if (!parents && B > B_old) return EL_ERR_INVALID_ARG;
    if (table_stride < columns || table_stride > ((int64_t)1 << 40) || out_of_reach(B_old, table_stride * 4)) return EL_ERR_INVALID_ARG;
    if (((uintptr_t)table | (uintptr_t)lengths | (uintptr_t)parents | (uintptr_t)counts | (uintptr_t)new_table | (uintptr_t)new_lengths | (uintptr_t)granted |
         (uintptr_t)copies | (uintptr_t)free_pages) & 3 || (uintptr_t)slots & 7) return EL_ERR_INVALID_ARG;
    const PlanSpace p = plan_space(B, pages);
    if (!workspace || workspace_bytes < p.total) return EL_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return EL_ERR_INVALID_ARG;
    char *const w = (char *)workspace;
    const PlanArgs a{table, table_stride, lengths, parents, counts, reserved, columns, B_old, pages, page_size, B, T, p.chunks, exclusive,
                     new_table, new_lengths, granted, copies, free_pages, slots, (Mark *)(w + p.marks), (int32_t *)(w + p.list), (int32_t *)(w + p.count),
                     (int64_t *)(w + p.before), (int64_t *)(w + p.block_need), (int32_t *)(w + p.need)};
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();      // errors other libraries left behind in this thread are not this launch's
    const int64_t work = (int64_t)B * columns + (int64_t)B * (slots ? T : T / page_size);
    if (pages <= kSmallPages && B <= kSmallLanes && work <= kSmallWork) {
        const int lds = pages * (int)(sizeof(Mark) + sizeof(int));
        hipLaunchKernelGGL(k_plan_small, dim3(1), dim3(kSmallLanes), lds, s, a);
        return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
    }
    const int clear = (pages + 1023) / 1024, parts = (columns + 4 * kLanes - 1) / (4 * kLanes), blocks = (B + kLanes - 1) / kLanes;
    hipLaunchKernelGGL(k_plan_clear, dim3(clear < 2048 ? clear : 2048), dim3(256), 0, s, a.marks, pages);
    hipLaunchKernelGGL(k_plan_mark, dim3(parts, B < 32768 ? B : 32768), dim3(kLanes), 0, s, a);
    hipLaunchKernelGGL(k_plan_count, dim3(p.chunks + blocks), dim3(kLanes), 0, s, a);
    hipLaunchKernelGGL(k_plan_assign, dim3(B + 1), dim3(kLanes), 0, s, a);
    return hipGetLastError() == hipSuccess ? EL_OK : EL_ERR_HIP;
}

} // namespace
} // namespace el

extern "C" size_t el_attn_plan_workspace_bytes(int32_t B, int32_t pages)
{
    if (B < 1 || B > el::kMaxSequences || pages < 1 || pages > el::kMaxPages) return 0;
    return el::plan_space(B, pages).total;
}

extern "C" el_status el_attn_plan_pages(const int32_t *table, int64_t table_stride, int32_t columns, const int32_t *lengths, int32_t B_old,
                                        const int32_t *parents, const int32_t *counts, const uint8_t *reserved, int32_t pages, int32_t page_size,
                                        int32_t B, int32_t T, int32_t *new_table, int32_t *new_lengths, int32_t *granted, int64_t *slots,
                                        int32_t *copies, int32_t *free_pages, void *workspace, size_t workspace_bytes, void *stream)
{
    return el::plan(false, table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T, new_table, new_lengths, granted,
                    slots, copies, free_pages, workspace, workspace_bytes, stream);
}

extern "C" el_status el_attn_plan_pages_exclusive(const int32_t *table, int64_t table_stride, int32_t columns, const int32_t *lengths, int32_t B_old,
                                                  const int32_t *parents, const int32_t *counts, const uint8_t *reserved, int32_t pages, int32_t page_size,
                                                  int32_t B, int32_t T, int32_t *new_table, int32_t *new_lengths, int32_t *granted, int64_t *slots,
                                                  int32_t *copies, int32_t *free_pages, void *workspace, size_t workspace_bytes, void *stream)
{
    return el::plan(true, table, table_stride, columns, lengths, B_old, parents, counts, reserved, pages, page_size, B, T, new_table, new_lengths, granted,
                    slots, copies, free_pages, workspace, workspace_bytes, stream);
}
