// Device code of page tables: pages handed out to sequences from a stack and taken back, and the slots of new tokens.
#pragma once

#include "equarx_device.hpp"

namespace equarx {
namespace pages {

struct Pool {
    Global<int32_t> table, lengths, free, free_count;
    int64_t width, pages;
    int32_t sequences, page;
};

// What a row is told: any may be null.
struct Rows {
    Global<int64_t> slots;
    Global<int32_t> positions, row_tags;
    Global<const int32_t> tags;
    int64_t rows;
};

constexpr int kTeam = 1024, kWaves = kTeam / 64;

// The sum of v over the threads before this one, and over all: every thread of the workgroup calls it.
struct Scan {
    int64_t before, all;
};

__device__ __forceinline__ Scan scan(int64_t v, int64_t *parts)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    __syncthreads();                    // parts may still be read from the scan before
    if (lane == 63) parts[wave] = sum;
    __syncthreads();
    Scan s{sum - v, 0};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) s.before += parts[i];
        s.all += parts[i];
    }
    return s;
}

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int32_t page) { return (tokens + page - 1) / page; }

// A sequence's tokens as the table can hold them.
__device__ __forceinline__ int64_t length_of(const Pool &p, int32_t b)
{
    const int64_t n = p.lengths[b], most = p.width * p.page;
    return n < 0 ? 0 : n < most ? n : most;
}

// The free pages that there are: the stack's own count, within its array.
__device__ __forceinline__ int64_t free_pages(const Pool &p)
{
    const int64_t n = p.free_count[0];
    return n < 0 ? 0 : n < p.pages ? n : p.pages;
}

// ---------------------------------------------------------------- back to a length

__global__ __launch_bounds__(kTeam) void trim_kernel(const Pool p, Global<const int32_t> keep)
{
    __shared__ int64_t parts[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t top = free_pages(p);
    // a wave a sequence, sixteen sequences at a time; pages to the stack in order of the sequences and of their tokens
    for (int32_t b0 = 0; b0 < p.sequences; b0 += kWaves) {
        const int32_t b = b0 + wave;
        const bool any = b < p.sequences;
        const int64_t n = any ? length_of(p, b) : 0, wanted = any ? keep[b] : 0, kept = wanted < 0 ? 0 : wanted < n ? wanted : n;
        const int64_t first = pages_of(kept, p.page), last = pages_of(n, p.page);
        int32_t *const row = p.table + (any ? b : 0) * p.width;
        auto is_page = [&](int64_t i) { return i < last && (uint32_t)row[i] < (uint64_t)p.pages; };
        int64_t count = 0;
        for (int64_t i0 = first; i0 < last; i0 += 64) count += __popcll(__ballot(is_page(i0 + lane)));
        const Scan s = scan(lane == 0 ? count : 0, parts);
        int64_t to = top + __shfl(s.before, 0);
        top += s.all;
        for (int64_t i0 = first; i0 < last; i0 += 64) {
            const int64_t i = i0 + lane;
            const bool real = is_page(i);
            const uint64_t mask = __ballot(real);
            const int64_t place = to + __popcll(mask & (((uint64_t)1 << lane) - 1));
            if (real && place < p.pages) p.free[place] = row[i];        // a page given back twice has no room at the last
            if (i < last) row[i] = -1;
            to += __popcll(mask);
        }
        if (any && lane == 0) p.lengths[b] = (int32_t)kept;
    }
    if (threadIdx.x == 0) p.free_count[0] = (int32_t)(top < p.pages ? top : p.pages);
}

// ---------------------------------------------------------------- new tokens

// What row `row` is told, q_starts and the table being complete; `count` the rows that are a sequence's.
__device__ __forceinline__ void tell_row(const Pool &p, const Rows &to, const int32_t *q_starts, const int32_t *lengths, int64_t row, int64_t count)
{
    int64_t slot = -1;
    int32_t position = -1, tag = -1;
    if (row < count) {
        int32_t lo = 0, hi = p.sequences;               // the last sequence that begins at or before the row
        while (hi - lo > 1) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (q_starts[mid] <= row) lo = mid; else hi = mid;
        }
        const int64_t t = lengths[lo] - (q_starts[lo + 1] - row);
        const int64_t entry = p.table[lo * p.width + t / p.page];
        if (entry >= 0 && entry < p.pages) slot = entry * p.page + t % p.page;
        position = (int32_t)t;
        if (to.row_tags.address) tag = to.tags[lo];
    }
    if (to.slots.address) to.slots[row] = slot;
    if (to.positions.address) to.positions[row] = position;
    if (to.row_tags.address) to.row_tags[row] = tag;
}

__global__ __launch_bounds__(kTeam) void extend_kernel(const Pool p, Global<const int32_t> counts, Global<int32_t> q_starts,
                                                          Global<int32_t> granted, const Rows to, int32_t tell)
{
    __shared__ int64_t parts[kWaves];
    const int64_t free = free_pages(p);
    int64_t rows = 0, wanted_pages = 0, taken = 0, granted_rows = 0;      // of the sequences before this thousand
    for (int32_t b0 = 0; b0 < p.sequences; b0 += kTeam) {
        const int32_t b = b0 + (int32_t)threadIdx.x;
        const bool any = b < p.sequences;
        const int64_t n = any ? length_of(p, b) : 0;
        int64_t want = any ? counts[b] : 0;
        if (want < 0 || n + want > p.width * p.page || n + want > INT32_MAX) want = 0;
        Scan s = scan(want, parts);
        if (rows + s.before + want > to.rows) want = 0;
        rows += s.all;
        const int64_t held = pages_of(n, p.page);
        int64_t need = pages_of(n + want, p.page) - held;
        s = scan(need, parts);
        const int64_t at = wanted_pages + s.before;
        wanted_pages += s.all;
        if (need > 0 && at + need > free) want = need = 0;
        s = scan(need, parts);
        taken += s.all;
        int32_t *const row = p.table + (any ? b : 0) * p.width;
        for (int64_t i = 0; i < need; ++i) row[held + i] = p.free[free - 1 - at - i];
        s = scan(want, parts);
        if (any) {
            q_starts[b] = (int32_t)(granted_rows + s.before);
            p.lengths[b] = (int32_t)(n + want);
            if (granted.address) granted[b] = (int32_t)want;
        }
        granted_rows += s.all;
    }
    if (threadIdx.x == 0) {
        q_starts[p.sequences] = (int32_t)granted_rows;
        p.free_count[0] = (int32_t)(free - taken);
    }
    if (!tell) return;
    __syncthreads();
    for (int64_t row = threadIdx.x; row < to.rows; row += kTeam) tell_row(p, to, q_starts, p.lengths, row, granted_rows);
}

__global__ __launch_bounds__(256) void tell_kernel(const Pool p, Global<const int32_t> q_starts, const Rows to)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row < to.rows) tell_row(p, to, q_starts, p.lengths, row, q_starts[p.sequences]);
}

}  // namespace pages
}  // namespace equarx
