// Device code of page tables: pages handed out to sequences from a stack and taken back, and the slots of new tokens.
#pragma once

#include "equarx_rows.hpp"

namespace equarx {
namespace pages {

struct Pool {
    Global<int32_t> table, lengths, free, free_count, seen;      // seen may be null
    int64_t width;
    int32_t pages, sequences, most;     // most: tokens that the table has room for, as far as a length can say it
    Divisor page;
};

// What a row is told: any but the slots may be null.
struct Rows {
    Global<int64_t> slots;
    Global<int32_t> positions, row_tags;
    Global<const int32_t> tags;
    int32_t rows;
};

constexpr int kTeam = 1024, kWaves = kTeam / 64;

// ---------------------------------------------------------------- sums over a workgroup
// Up to 2^30 + 1, at which a sum stays: more than rows or pages there can be is as much as one more.

constexpr uint32_t kMany = (1u << 30) + 1;

__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return a + b < kMany ? a + b : kMany; }

__device__ __forceinline__ uint32_t wave_scan(uint32_t v)
{
    return equarx::wave_scan(v, [](uint32_t a, uint32_t b) { return add(a, b); });
}

struct Scan {
    uint32_t upto, all;         // this thread's and those before it; all threads'
};

// N sums at once, with two barriers; every thread of the workgroup calls it.
template <int N>
__device__ __forceinline__ void scan(const uint32_t (&v)[N], Scan (&s)[N], uint32_t (*parts)[kWaves])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i].upto = wave_scan(v[i]);
    __syncthreads();                            // the last scan's parts have been read
    if (lane == 63) {
#pragma unroll
        for (int i = 0; i < N; ++i) parts[i][wave] = s[i].upto;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t upto = wave_scan(lane < kWaves ? parts[i][lane] : 0);
        s[i].all = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWaves - 1);
        if (wave > 0) s[i].upto = add(s[i].upto, (uint32_t)__builtin_amdgcn_readlane((int)upto, wave - 1));
    }
}

// ---------------------------------------------------------------- numbers as they are taken

__device__ __forceinline__ int32_t pages_of(const Pool &p, int32_t tokens) { return tokens > 0 ? (int32_t)p.page.of((uint32_t)tokens - 1) + 1 : 0; }

__device__ __forceinline__ int32_t within(int32_t v, int32_t most) { return v < 0 ? 0 : v < most ? v : most; }

__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// The last i of [0, n) with from[i] <= at, from[0] being one.
template <typename T>
__device__ __forceinline__ int32_t last_from(const T *from, int32_t n, uint32_t at)
{
    int32_t lo = 0;
    for (int32_t step = 1 << 20; step > 0; step /= 2) {
        if (step < n && lo + step < n && (uint32_t)from[lo + step] <= at) lo += step;
    }
    return lo;
}

// ---------------------------------------------------------------- back to a length
// Latency is all there is to it: a thread a sequence for what is given back, then a thread an entry, 1024 at a time.

__global__ __launch_bounds__(kTeam) void trim_kernel(const Pool p, Global<const int32_t> keep)
{
    __shared__ uint32_t parts[1][kWaves], from[kTeam];
    __shared__ int32_t first_of[kTeam];
    const int i = threadIdx.x;
    int64_t top = within(p.free_count[0], p.pages);
    for (int32_t b0 = 0; b0 < p.sequences; b0 += kTeam) {
        const int32_t b = b0 + i, here = p.sequences - b0 < kTeam ? p.sequences - b0 : kTeam;
        int32_t n = 0, kept = 0;
        if (b < p.sequences) {
            n = within(p.lengths[b], p.most);
            kept = within(keep[b], n);
        }
        const int32_t first = pages_of(p, kept), last = pages_of(p, n);
        const uint32_t gone[1] = {(uint32_t)(last - first)};
        Scan s[1];
        scan(gone, s, parts);
        from[i] = s[0].upto - gone[0];
        first_of[i] = first;
        if (b < p.sequences) p.lengths[b] = kept;
        const uint32_t all = s[0].all;
        __syncthreads();
        for (uint32_t e0 = 0; e0 < all; e0 += kTeam) {
            const uint32_t e = e0 + i;
            int32_t page = -1;
            if (e < all) {
                const int32_t q = last_from(from, here, e);
                int32_t *const entry = p.table + (int64_t)(b0 + q) * p.width + first_of[q] + (e - from[q]);
                page = *entry;
                *entry = -1;
            }
            const uint32_t real[1] = {(uint32_t)page < (uint32_t)p.pages ? 1u : 0u};
            scan(real, s, parts);
            const int64_t place = top + s[0].upto - 1;
            if (real[0] && place < p.pages) p.free[place] = page;       // a page given back twice has no room at the last
            top += s[0].all;
        }
        __syncthreads();
    }
    if (i == 0) p.free_count[0] = (int32_t)(top < p.pages ? top : p.pages);
}

// ---------------------------------------------------------------- new tokens

// What row `row` of sequence b is told: `begin` the sequence's first row, `n` its tokens before the step.
__device__ __forceinline__ void tell_row(const Pool &p, const Rows &to, int32_t row, int32_t b, int32_t begin, int32_t n)
{
    const int32_t t = n + row - begin, at = (int32_t)p.page.of((uint32_t)t), page = (int32_t)p.page.d;
    const int32_t entry = p.table[b * p.width + at];
    to.slots[row] = (uint32_t)entry < (uint32_t)p.pages ? (int64_t)entry * page + (t - at * page) : -1;
    if (to.positions.address) to.positions[row] = t;
    if (to.row_tags.address) to.row_tags[row] = to.tags[b];
}

__device__ __forceinline__ void tell_nothing(const Rows &to, int32_t row)
{
    to.slots[row] = -1;
    if (to.positions.address) to.positions[row] = -1;
    if (to.row_tags.address) to.row_tags[row] = -1;
}

// One workgroup decides and hands out.  A thread a sequence; one scan says what all of them want, and if rows and stack have it, that is
// what they get; else two more say who goes without.  Then a thread an entry of the table, and, with `tell`, a thread a row.  Where rows
// stay as they were asked for (p.seen), those before a sequence come from its neighbour: sums that stay at kMany are no differences.
__global__ __launch_bounds__(kTeam) void extend_kernel(const Pool p, Global<const int32_t> counts, Global<int32_t> q_starts,
                                                       Global<int32_t> granted, const Rows to, int32_t tell)
{
    __shared__ uint32_t parts[2][kWaves], from[kTeam];
    __shared__ int32_t held_of[kTeam], begin_of[kTeam], had[kTeam];
    const int i = threadIdx.x;
    const int32_t free = p.sequences > 0 ? within(p.free_count[0], p.pages) : 0;       // without sequences there need be no pages
    const bool stay = p.seen.address != 0;
    uint32_t rows = 0, pages = 0, got_rows = 0;          // wanted by the sequences before these 1024, and got (or, if they stay, had)
    int32_t taken = 0;
    for (int32_t b0 = 0; b0 < p.sequences; b0 += kTeam) {
        const int32_t b = b0 + i, here = p.sequences - b0 < kTeam ? p.sequences - b0 : kTeam;
        const uint32_t first_row = got_rows;
        int32_t n = 0;
        uint32_t want = 0, asked = 0;
        if (b < p.sequences) {
            n = within(p.lengths[b], p.most);
            const int32_t count = counts[b];
            if (count > 0 && count <= p.most - n) want = (uint32_t)count;
            asked = stay ? (uint32_t)within(count, (int32_t)kMany) : want < kMany ? want : kMany;
        }
        const int32_t held = pages_of(p, n);
        uint32_t need = (uint32_t)(pages_of(p, n + (int32_t)want) - held);
        Scan s[2];
        scan<2>({asked, need}, s, parts);
        uint32_t begin = got_rows + s[0].upto - asked;                 // with all of them served
        const bool enough = rows == got_rows && pages == (uint32_t)taken && add(rows, s[0].all) <= (uint32_t)to.rows &&
                            add(pages, s[1].all) <= (uint32_t)free;
        if (enough) {
            rows = got_rows = rows + s[0].all;
            pages += s[1].all;
            taken = (int32_t)pages;
        } else {
            const uint32_t rows_upto = add(rows, s[0].upto);
            uint32_t before = 0;
            if (stay) {
                from[i] = rows_upto;
                __syncthreads();
                before = i > 0 ? from[i - 1] : rows;
            }
            rows = add(rows, s[0].all);
            if (rows_upto > (uint32_t)to.rows) want = need = 0;
            Scan some[1];
            scan<1>({need}, some, parts);
            const uint32_t pages_upto = add(pages, some[0].upto);
            pages = add(pages, some[0].all);
            if (need > 0 && pages_upto > (uint32_t)free) want = need = 0;
            scan<2>({want, need}, s, parts);
            begin = stay ? umin(before, (uint32_t)to.rows) : got_rows + s[0].upto - want;
            got_rows = stay ? umin(rows, (uint32_t)to.rows) : got_rows + s[0].all;
            taken += (int32_t)s[1].all;
        }
        if (b < p.sequences) {
            q_starts[b] = (int32_t)begin;
            p.lengths[b] = n + (int32_t)want;
            if (granted.address) granted[b] = (int32_t)want;
            if (stay) p.seen[b] = asked > 0 && want == 0 ? 0 : n + (int32_t)want;
        }
        from[i] = s[1].upto - need;                     // of the entries that are handed out here
        held_of[i] = held;
        begin_of[i] = (int32_t)begin;
        had[i] = want > 0 ? n : -1;
        // the first entry's page: those before are the sequences' before these
        const int32_t top = free - 1 - (taken - (int32_t)s[1].all);
        const uint32_t all = s[1].all;
        __syncthreads();
        for (uint32_t e = i; e < all; e += kTeam) {
            const int32_t q = last_from(from, here, e);
            p.table[(int64_t)(b0 + q) * p.width + held_of[q] + (e - from[q])] = p.free[top - (int32_t)e];
        }
        __syncthreads();
        if (tell) {
            for (uint32_t row = first_row + i; row < got_rows; row += kTeam) {
                const int32_t q = last_from(begin_of, here, row);
                if (had[q] < 0) {
                    tell_nothing(to, (int32_t)row);
                } else {
                    tell_row(p, to, (int32_t)row, b0 + q, begin_of[q], had[q]);
                }
            }
            __syncthreads();
        }
    }
    if (i == 0) {
        q_starts[p.sequences] = (int32_t)got_rows;
        if (p.sequences > 0) p.free_count[0] = free - taken;
    }
    if (tell) {
        for (int32_t row = (int32_t)got_rows + i; row < to.rows; row += kTeam) tell_nothing(to, row);
    }
}

// Many rows, by workgroups of their own; the sequences' first rows come to LDS where they fit.
__global__ __launch_bounds__(256) void tell_kernel(const Pool p, Global<const int32_t> q_starts, const Rows to)
{
    constexpr int kFit = 1024;
    __shared__ int32_t starts[kFit];
    const int32_t row = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    const int32_t all = q_starts[p.sequences];
    const bool fits = p.sequences <= kFit;
    if (fits) {
        for (int32_t i = threadIdx.x; i < p.sequences; i += 256) starts[i] = q_starts[i];
        __syncthreads();
    }
    if (row >= to.rows) return;
    if (row >= all) {
        tell_nothing(to, row);
        return;
    }
    const int32_t b = fits ? last_from(starts, p.sequences, (uint32_t)row) : last_from((const int32_t *)q_starts, p.sequences, (uint32_t)row);
    const int32_t begin = q_starts[b], now = p.seen.address ? p.seen[b] : p.lengths[b];
    if (now == 0) {
        tell_nothing(to, row);
        return;
    }
    tell_row(p, to, row, b, begin, now - (q_starts[b + 1] - begin));
}

}  // namespace pages
}  // namespace equarx
