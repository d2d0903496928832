// Device code of low-rank adapters of many requests: rows brought together by adapter, t = A x, and out += f B t.
#pragma once

#include <type_traits>

#include "equarx.h"
#include "equarx_rows.hpp"

namespace equarx {
namespace adapters {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMostSlices = EQUARX_ADAPTERS_MAX_SLICES, kMostAdapters = EQUARX_ADAPTERS_MAX;

// Rows of one adapter that are taken together: item i has `count` rows, order[i * tile] and on, tile of them at most.
struct Item {
    int32_t adapter, count;
};

// ---------------------------------------------------------------- rows by adapter
// One workgroup counts, lays out and places.  Which of an adapter's rows comes first is left to the atomics: a row's results are its
// own column of the products below and do not depend on its place.

// at[a] += 1 for every lane with 0 <= a < adapters; returns what each found, the lanes of one adapter one after the other.  Lanes with the same
// adapter as the first of those left wait for each other in the atomics: four times they are added as one.
__device__ __forceinline__ int32_t count_up(int32_t *at, int32_t a, int32_t adapters)
{
    const int lane = threadIdx.x & 63;
    bool left = a >= 0 && a < adapters;
    int32_t found = 0;
    for (int i = 0; i < 4; ++i) {
        const uint64_t mask = __ballot(left);
        if (mask == 0) return found;
        const int first = __builtin_ctzll(mask);
        const uint64_t same = __ballot(left && a == __builtin_amdgcn_readlane(a, first));
        if (same >> lane & 1) left = false;
        int32_t base = 0;
        if (lane == first) base = atomicAdd(&at[a], (int32_t)__popcll(same));
        base = __builtin_amdgcn_readlane(base, first);
        if (same >> lane & 1) found = base + (int32_t)__popcll(same & (((uint64_t)1 << lane) - 1));
    }
    if (left) found = atomicAdd(&at[a], 1);
    return found;
}

__device__ __forceinline__ int32_t wave_sums(int32_t v)
{
    return (int32_t)wave_scan((uint32_t)v, [](uint32_t a, uint32_t b) { return a + b; });
}

__global__ __launch_bounds__(1024) void group_kernel(Global<const int32_t> ids, int32_t M, int32_t adapters, int32_t tile, Global<int32_t> order,
                                                     Global<Item> items, int32_t most_items)
{
    __shared__ int32_t at[kMostAdapters];
    __shared__ int32_t parts[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kKept = 8;                                    // ids of a thread that are asked for together, and kept where they are all
    int32_t kept[kKept];
    auto load = [&](int32_t m0) {
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            const int32_t m = m0 + i * 1024 + (int32_t)threadIdx.x;
            kept[i] = m < M ? ids[m] : -1;
        }
    };
    load(0);
    for (int a = threadIdx.x; a < adapters; a += 1024) at[a] = 0;
    __syncthreads();
    for (int32_t m0 = 0; m0 < M; m0 += kKept * 1024) {
        if (m0 > 0) load(m0);
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            if (m0 + i * 1024 < M) count_up(at, kept[i], adapters);
        }
    }
    __syncthreads();
    int32_t done = 0;
    for (int a0 = 0; a0 < adapters; a0 += 1024) {
        const int a = a0 + (int)threadIdx.x;
        const int32_t n = a < adapters ? at[a] : 0, pieces = (n + tile - 1) / tile;
        const int32_t p = wave_sums(pieces);
        __syncthreads();
        if (lane == 63) parts[wave] = p;
        __syncthreads();
        int32_t item = done + p - pieces;
        for (int i = 0; i < 16; ++i) {
            if (i < wave) item += parts[i];
            done += parts[i];
        }
        if (a < adapters) at[a] = item * tile;
        for (int32_t i = 0; i < pieces; ++i) items[item + i] = Item{a, n - i * tile < tile ? n - i * tile : tile};
    }
    for (int32_t i = done + (int32_t)threadIdx.x; i < most_items; i += 1024) items[i] = Item{0, 0};
    __syncthreads();
    for (int32_t m0 = 0; m0 < M; m0 += kKept * 1024) {
        if (M > kKept * 1024) load(m0);
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            if (m0 + i * 1024 >= M) break;
            const int32_t place = count_up(at, kept[i], adapters);
            if (kept[i] >= 0 && kept[i] < adapters) order[place] = m0 + i * 1024 + (int32_t)threadIdx.x;
        }
    }
}

// What lanes of a wave hand each other through LDS needs no barrier, but the compiler has to leave it in order.
__device__ __forceinline__ void in_wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Few rows are brought together without a launch: item i is row i's, if every sixteenth of its adapter's rows, from the first on, is row i,
// and has that row and the next fifteen.  Each wave finds that for itself, with lane l's rows l, 64 + l, ...
constexpr int kFewRows = 256, kIdsPerLane = kFewRows / 64;

// Row l % 16 of item i in lane l; `count` rows, 0 where there is no such item.
__device__ __forceinline__ int32_t find_item(const int32_t *ids, int32_t M, int32_t adapters, int32_t i, int32_t *places, Item &item)
{
    const int lane = threadIdx.x & 63;
    int32_t id[kIdsPerLane];
#pragma unroll
    for (int q = 0; q < kIdsPerLane; ++q) id[q] = q * 64 + lane < M ? ids[q * 64 + lane] : -1;
    const int32_t mine = ids[i];
    int32_t before = 0, all = 0, rank[kIdsPerLane];
#pragma unroll
    for (int q = 0; q < kIdsPerLane; ++q) {
        const uint64_t same = __ballot(id[q] == mine);
        const int32_t left = i - q * 64;                        // rows of these that come before row i
        const uint64_t lower = left <= 0 ? 0 : left >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << left) - 1;
        before += __popcll(same & lower);
        rank[q] = all + __popcll(same & (((uint64_t)1 << lane) - 1));
        all += __popcll(same);
    }
    item = Item{mine, all - before < 16 ? all - before : 16};
    if (mine < 0 || mine >= adapters || before % 16 != 0) item.count = 0;
#pragma unroll
    for (int q = 0; q < kIdsPerLane; ++q) {
        if (id[q] == mine && rank[q] >= before && rank[q] < before + 16) places[rank[q] - before] = q * 64 + lane;
    }
    in_wave_order();
    return places[lane % 16 < item.count ? lane % 16 : 0];
}

// More rows, without a launch too: every workgroup counts all of them, finds what its item is, and which rows that has, in their order: every
// workgroup has to find the same.  T rows of an item at most; W waves, of which each has rows that follow each other, I a lane at most.
constexpr int kFoundAdapters = 1024;

template <int T, int W, int I>
__device__ __forceinline__ void find_rows(const int32_t *ids, int32_t M, int32_t adapters, int32_t i, int32_t *at, int32_t *places, Item &item)
{
    __shared__ int32_t parts[2][W], found[3];
    constexpr int kEach = kFoundAdapters / (64 * W);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t per = (M + 64 * W - 1) / (64 * W), m0 = wave * per * 64 + lane;
    int32_t id[I];
#pragma unroll
    for (int q = 0; q < I; ++q) id[q] = q < per && m0 + q * 64 < M ? ids[m0 + q * 64] : -1;
    for (int a = threadIdx.x; a < kFoundAdapters; a += 64 * W) at[a] = 0;
    if (threadIdx.x == 0) found[2] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < I; ++q) {
        if (q < per) count_up(at, id[q], adapters);
    }
    __syncthreads();
    int32_t n[kEach], pieces = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        n[e] = at[threadIdx.x * kEach + e];
        pieces += (n[e] + T - 1) / T;
    }
    const int32_t upto = wave_sums(pieces);
    if (lane == 63) parts[0][wave] = upto;
    __syncthreads();
    int32_t first = upto - pieces;
    for (int w = 0; w < wave; ++w) first += parts[0][w];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int32_t next = first + (n[e] + T - 1) / T;
        if (first <= i && i < next) {
            found[0] = threadIdx.x * kEach + e;
            found[1] = (i - first) * T;
            found[2] = n[e] - (i - first) * T < T ? n[e] - (i - first) * T : T;
        }
        first = next;
    }
    __syncthreads();
    item = Item{__builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[2])};
    if (item.count == 0) return;
    uint64_t same[I];
    int32_t all = 0;
#pragma unroll
    for (int q = 0; q < I; ++q) {
        same[q] = __ballot(id[q] == item.adapter);
        all += __popcll(same[q]);
    }
    if (lane == 0) parts[1][wave] = all;
    __syncthreads();
    int32_t place = -found[1];
    for (int w = 0; w < wave; ++w) place += parts[1][w];
#pragma unroll
    for (int q = 0; q < I; ++q) {
        const int32_t mine = place + (int32_t)__popcll(same[q] & (((uint64_t)1 << lane) - 1));
        if (id[q] == item.adapter && mine >= 0 && mine < T) places[mine] = m0 + q * 64;
        place += __popcll(same[q]);
    }
    __syncthreads();
}

// ---------------------------------------------------------------- products of sixteen by sixteen
// v_mfma_f32_16x16x32_bf16: lane l has row l % 16 of the first operand and column l % 16 of the second, k = 8 (l / 16) + 0 .. 7 of both,
// and of the result column l % 16, rows 4 (l / 16) + 0 .. 3.  Rows of x are always the columns: a NaN or an infinity stays in its row.

__device__ __forceinline__ v4f multiply(const u32x4 &a, const u32x4 &b, const v4f &sum)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), sum, 0, 0, 0);
}

__device__ __forceinline__ u32x4 load8(const uint16_t *p) { return *reinterpret_cast<const u32x4_anywhere *>(p); }

// A lane's operand is sixteen bytes of a row, its neighbour's of the next row: loaded so, every lane is an access of the cache by itself (four a
// cycle at 64 bytes a lane's quad would be one), and those bounded both kernels (4096 rows, rank 64: 18 and 32 us).  So rows come in whole
// 128 bytes, eight lanes a row, and through LDS to the lanes that multiply; each wave has a place of its own there, and no barrier is needed.

// Items of one adapter, which follow each other, go to one XCD, and all XCDs have as many: `together` items, as many as an adapter has in the mean, are one
// XCD's, the next the next one's.  Workgroups go round the eight: which item `x` of `count` (a multiple of eight) is.
__device__ __forceinline__ int32_t item_of(uint32_t x, uint32_t count, uint32_t together)
{
    const uint32_t turns = x / (8 * together) * (8 * together), each = turns + 8 * together <= count ? together : (count - turns) / 8;
    return (int32_t)(turns + (x & 7) * each + (x - turns) / 8);
}

// ---------------------------------------------------------------- t = A x
// A workgroup has an item's rows or one of Parts of them, 16 RT, 16 QT rows of A and a piece of k, of which its W waves take 64 in turn; their sums are
// added in order through LDS.  Sums of the pieces go to t [split][M][R].  A wave's next step is on its way
// while it multiplies one; a second gained nothing.  64 rows of 32 adapters, 48 x 5376: 6.2 us, 2.7 TB/s of A; 4096 rows of 4, 64 x 5376: 14.3 without
// what finds the rows (3 more), the 44 MB of x at 3.1 TB/s, of which a workgroup has a CU's LDS and 128 KB on their way.
// kFind: items are found here, and the first workgroup of each writes it down for the launch that follows.

constexpr int kStep = 64;

// How an item is found: few rows, by a list, or, with so many rows a lane, among all.
enum Find { kFew = -1, kListed = 0, kFound = 8, kFoundLong = 16 };

template <int RT, int QT, int W, int Parts, Find kFind>
__global__ __launch_bounds__(64 * W) void shrink_kernel(Global<const uint16_t> x, int64_t x_stride, Global<const uint16_t> a, Global<float> t,
                                                        int32_t M, int32_t K, int32_t R, int32_t piece, Global<int32_t> order, Global<Item> items,
                                                        Global<const int32_t> ids, int32_t adapters, int32_t together)
{
    constexpr int T = 16 * RT, Q = 16 * QT, kPitch = Q + 4, kTile = (T + Q) * 2 * kStep;
    constexpr int kSums = W * 16 * kPitch * 4, kAll = W * kTile > kSums ? W * kTile : kSums;
    __shared__ __align__(16) uint8_t lds[kAll];
    __shared__ int32_t places[kFind == kFew ? W : 1][kFind == kListed ? 1 : T * Parts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int32_t index = kFind == kFew ? (int32_t)blockIdx.x : item_of(blockIdx.x, gridDim.x, together), at = index / Parts, part = index % Parts;
    Item item;
    if constexpr (kFind == kFew) {
        const int32_t row = find_item(ids, M, adapters, at, places[wave], item);
        if (blockIdx.y == 0 && blockIdx.z == 0 && wave == 0) {
            if (lane == 0) items[at] = item;
            if (lane < item.count) order[at * 16 + lane] = row;
        }
    } else if constexpr (kFind != kListed) {
        static_assert(kFoundAdapters * 4 <= kAll, "counts have the operands' place");
        find_rows<T * Parts, W, kFind>(ids, M, adapters, at, reinterpret_cast<int32_t *>(lds), places[0], item);
        if (part == 0 && blockIdx.y == 0 && blockIdx.z == 0 && wave == 0) {
            if (lane == 0) items[at] = item;
            if (lane < item.count) order[at * (T * Parts) + lane] = places[0][lane];
        }
    } else {
        item = items[at];
    }
    item.count = item.count - part * T < T ? item.count - part * T : T;
    if (item.count <= 0) return;
    const int32_t *const rows = (kFind == kFew ? places[wave] : kFind != kListed ? places[0] : (const int32_t *)order + (int64_t)at * (T * Parts)) + part * T;
    const int32_t r0 = blockIdx.y * Q, k_from = blockIdx.z * piece, k_to = k_from + piece < K ? k_from + piece : K;
    const int in = lane / 8, eighth = lane % 8;                 // of the rows that are loaded
    const uint16_t *from[2 * (RT + QT)];
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) from[i] = x + rows[i * 8 + in < item.count ? i * 8 + in : 0] * x_stride;
#pragma unroll
    for (int i = 0; i < 2 * QT; ++i) {
        const int32_t r = r0 + i * 8 + in < R ? r0 + i * 8 + in : R - 1;
        from[2 * RT + i] = a + ((int64_t)item.adapter * R + r) * K;
    }
    struct Step {
        u32x4 v[2 * (RT + QT)];
    };
    uint8_t *const mine = lds + wave * kTile;
    auto put = [&](const Step &s) {                             // block b of row r in place b xor r / 2 % 8: sixteen rows' block is in all banks
#pragma unroll
        for (int i = 0; i < 2 * (RT + QT); ++i) {
            const int row = i * 8 + in;
            *reinterpret_cast<u32x4 *>(mine + row * (2 * kStep) + (eighth ^ (row >> 1 & 7)) * 16) = s.v[i];
        }
        in_wave_order();
    };
    v4f sum[RT][QT] = {};
    auto add = [&]() {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            u32x4 av[QT];
            auto get = [&](int row) { return *reinterpret_cast<const u32x4 *>(mine + row * (2 * kStep) + ((j * 4 + g) ^ (row >> 1 & 7)) * 16); };
#pragma unroll
            for (int q = 0; q < QT; ++q) av[q] = get(T + q * 16 + l);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const u32x4 xv = get(i * 16 + l);
#pragma unroll
                for (int q = 0; q < QT; ++q) sum[i][q] = multiply(av[q], xv, sum[i][q]);
            }
        }
        in_wave_order();
    };
    // Whole steps; no load is behind a condition (behind one the compiler waits for it there): past the last it is the last once more, not added.
    const int32_t steps = (k_to - k_from) / kStep;
    auto whole = [&](Step &to, int32_t step) {
        const int32_t k = k_from + (step < steps ? step : steps - 1) * kStep + eighth * 8;
#pragma unroll
        for (int i = 0; i < 2 * (RT + QT); ++i) to.v[i] = load8(from[i] + k);
    };
    if (wave < steps) {
        Step now;
        whole(now, wave);
        for (int32_t step = wave; step < steps; step += W) {
            put(now);
            whole(now, step + W);
            add();
        }
    }
    if (k_from + steps * kStep < k_to && steps % W == wave) {      // past K zeros, in both
        Step last;
        const int32_t k = k_from + steps * kStep + eighth * 8;
#pragma unroll
        for (int i = 0; i < 2 * (RT + QT); ++i) last.v[i] = K >= 8 ? load_row8_back(from[i], k, K) : load_row8(from[i], k, K);
        put(last);
        add();
    }
    float(*const sums)[16][kPitch] = reinterpret_cast<float(*)[16][kPitch]>(lds);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < QT; ++q) *reinterpret_cast<v4f *>(&sums[wave][l][q * 16 + g * 4]) = sum[i][q];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * QT * 4; e += 64 * W) {
            const int row = e / (QT * 4), r = e % (QT * 4) * 4;
            if (i * 16 + row >= item.count || r0 + r >= R) continue;            // R is a multiple of 8
            v4f v = *reinterpret_cast<const v4f *>(&sums[0][row][r]);
#pragma unroll
            for (int w = 1; w < W; ++w) v += *reinterpret_cast<const v4f *>(&sums[w][row][r]);
            *reinterpret_cast<v4f *>(t + ((int64_t)blockIdx.z * M + rows[i * 16 + row]) * R + r0 + r) = v;
        }
    }
}

// ---------------------------------------------------------------- out += f B t
// t, joined from its partial sums, is taken as two bf16 and stays in registers; B's columns come to LDS and meet both halves; what comes of sixteen
// rows and 64 columns goes through LDS to the lanes that have eight columns of a row.  S: steps of 32 of the rank, at most.  kNarrow: rows of fewer
// than eight columns.  kStreams: out is more than the caches keep for the next call, and is read and written past them.

struct Slices {
    int32_t first_column[kMostSlices + 1], first_chunk[kMostSlices + 1];     // of the slices there are; the end after them
};

// What a launch hands to its workgroups.
struct Expansion {
    Global<uint16_t> out;
    int64_t out_stride;
    Global<const uint16_t> b;
    Global<const float> factors, t;
    int32_t M, N, rank, slices, splits, chunks, together;
    Global<const int32_t> order;
    Global<const Item> items;
    Slices cut;
};

// bytes of a column of B in LDS, with a shift of banks, and of a row of 64 results
template <int S>
constexpr int kColumn = S * 64 + 16;
constexpr int kResult = 64 * 4 + 16;

constexpr float kMostBf16 = 0x1.fep127f;

// A wave's sixteen rows of an item.
template <int S, bool kNarrow, bool kStreams>
struct SixteenRows {
    int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, in = lane / 8, eighth = lane % 8;
    int32_t count, N;
    float after;                // what of the factor the sums are multiplied by
    uint16_t *row[2];
    u32x4 t[2 * S];
    struct Before {
        u32x4 v[2];
    };

    int32_t place[2], mine;

    // The rows' numbers are asked for beside the item: behind its last they are whatever the place holds, and not used.
    __device__ __forceinline__ SixteenRows(const Expansion &p, const int32_t *rows) : N(p.N)
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) place[half] = rows[half * 8 + in];
        mine = rows[l];
    }

    __device__ __forceinline__ void take(const Expansion &p, int32_t count_)
    {
        count = count_;
        const int32_t first = __builtin_amdgcn_readfirstlane(mine);
#pragma unroll
        for (int half = 0; half < 2; ++half) row[half] = p.out + (half * 8 + in < count ? place[half] : first) * p.out_stride;
        mine = l < count ? mine : first;
    }

    // What is added to.  No load is behind a condition (the compiler waits for what it loads there): rows that are not there are the first once more, and
    // units that reach past a row's end begin before it (drop_elements puts their elements in place).
    __device__ __forceinline__ void load(Before &to, int32_t n0) const
    {
        const int32_t n = n0 + eighth * 8;
#pragma unroll
        for (int half = 0; half < 2; ++half) if constexpr (kNarrow) {
                to.v[half] = load_row8(row[half], n, N);
            } else {
                const auto *const from = reinterpret_cast<const u32x4_anywhere *>(row[half] + (n + 8 <= N ? n : N - 8));
                to.v[half] = kStreams ? __builtin_nontemporal_load(from) : *from;
            }
    }

    // The rows' t of slice s: lane l has row l % 16, eight entries of each step.  A factor below one is multiplied to t, where sums of B t might
    // pass fp32's range and their product with it not; another to the sums (`after`), where its product with t might.  The larger half of t is
    // bf16's largest where rounding would make it infinite, and the smaller one the rest: of an infinity an infinity, of a NaN a NaN.
    __device__ __forceinline__ void join(const Expansion &p, int s, float factor)
    {
        const bool below = __builtin_fabsf(factor) < 1.0f;
        const float ahead = below ? factor : 1.0f;
        after = below ? 1.0f : factor;
        const int32_t R = p.slices * p.rank;
        const float *const from = p.t + (int64_t)mine * R + s * p.rank;
        // in order, and several asked for together: one after the other is a latency each
        v4f v[S][2] = {};
        auto several = [&](auto most, int32_t i) {
            constexpr int J = decltype(most)::value;
            v4f part[J][S][2];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float *const at = from + (int64_t)(i + j < p.splits ? i + j : i) * p.M * R;
#pragma unroll
                for (int q = 0; q < S; ++q) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int32_t k = q * 32 + g * 8 + h * 4;
                        part[j][q][h] = *reinterpret_cast<const v4f *>(at + (k < p.rank ? k : 0));
                    }
                }
            }
            asm volatile("" ::: "memory");                      // or they move to the additions, each behind its condition
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if (j > 0 && i + j >= p.splits) break;
#pragma unroll
                for (int q = 0; q < S; ++q) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) v[q][h] = i + j == 0 ? part[j][q][h] : v[q][h] + part[j][q][h];
                }
            }
        };
        if (p.splits <= 2) {
            several(std::integral_constant<int, 2>{}, 0);
        } else {
            constexpr int kMany = S <= 2 ? 4 : 2;
            for (int32_t i = 0; i < p.splits; i += kMany) several(std::integral_constant<int, kMany>{}, i);
        }
#pragma unroll
        for (int q = 0; q < S; ++q) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4f f = q * 32 + g * 8 < p.rank ? v[q][h] * ahead : v4f{0, 0, 0, 0};
                float w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_fmed3f(f[i], -kMostBf16, kMostBf16);
                const u32x2 high = {narrow_bf16x2(w[0], w[1]), narrow_bf16x2(w[2], w[3])};
                widen_bf16x4(high, w);
                const u32x2 low = {narrow_bf16x2(f[0] - w[0], f[1] - w[1]), narrow_bf16x2(f[2] - w[2], f[3] - w[3])};
                t[q][2 * h] = high.x;
                t[q][2 * h + 1] = high.y;
                t[S + q][2 * h] = low.x;
                t[S + q][2 * h + 1] = low.y;
            }
        }
    }

    __device__ __forceinline__ void multiply_columns(const uint8_t *columns, v4f (&sum)[4]) const
    {
#pragma unroll
        for (int q = 0; q < S; ++q) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sum[i] = multiply(*reinterpret_cast<const u32x4 *>(columns + (i * 16 + l) * kColumn<S> + q * 64 + g * 16), t[q], sum[i]);
        }
#pragma unroll
        for (int q = 0; q < S; ++q) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sum[i] = multiply(*reinterpret_cast<const u32x4 *>(columns + (i * 16 + l) * kColumn<S> + q * 64 + g * 16), t[S + q], sum[i]);
        }
    }

    // Sums of the columns from n0 on, through `results`, to the rows, as far as n_end.
    __device__ __forceinline__ void store(const v4f (&sum)[4], const Before &before, uint8_t *results, int32_t n0, int32_t n_end) const
    {
        const int32_t n = n0 + eighth * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<v4f *>(results + l * kResult + (i * 16 + g * 4) * 4) = sum[i];
        in_wave_order();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint8_t *const p = results + (half * 8 + in) * kResult + eighth * 32;
            const v4f d[2] = {*reinterpret_cast<const v4f *>(p), *reinterpret_cast<const v4f *>(p + 16)};
            float f[8];
            widen_bf16x8(kNarrow || n + 8 <= N ? before.v[half] : drop_elements(before.v[half], n + 8 - N), f);
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = narrow_bf16x2(__builtin_fmaf(d[i / 2][i % 2 * 2], after, f[2 * i]), __builtin_fmaf(d[i / 2][i % 2 * 2 + 1], after, f[2 * i + 1]));
            if (n0 + 64 <= n_end) {                             // all of the wave's columns
                auto *const to = reinterpret_cast<u32x4_anywhere *>(row[half] + n);
                if (half * 8 + in < count) {
                    if constexpr (kStreams) {
                        __builtin_nontemporal_store(v, to);
                    } else {
                        *to = v;
                    }
                }
            } else if (half * 8 + in < count && n < n_end) {
                store_row8(row[half], n, n_end, v);
            }
        }
        in_wave_order();
    }
};

// 64 columns of B on their way to LDS by Threads lanes: pieces of eight of the rank, one after the other as they lie in memory.
template <int S, int Threads>
struct Columns {
    static constexpr int kPieces = 64 * 4 * S / Threads;
    u32x4 v[kPieces];

    __device__ __forceinline__ void load(const uint8_t *adapter, uint32_t per, int32_t n0, int32_t n_end)      // 2^30 bytes at most
    {
        const uint32_t last = (uint32_t)n_end * per - 1;        // past the slice's end it is the last piece once more
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t e = (uint32_t)n0 * per + i * Threads + threadIdx.x % Threads;
            v[i] = *reinterpret_cast<const u32x4 *>(adapter + (e < last ? e : last) * 16);
        }
    }

    __device__ __forceinline__ void put(uint8_t *columns, uint32_t per) const
    {
        const uint32_t thread = threadIdx.x % Threads;
        if (per == 4 * S) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint32_t e = i * Threads + thread;
                *reinterpret_cast<u32x4 *>(columns + e / (4 * S) * kColumn<S> + e % (4 * S) * 16) = v[i];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t e = i * Threads + thread, c = e / per;
            if (c < 64) *reinterpret_cast<u32x4 *>(columns + c * kColumn<S> + (e - c * per) * 16) = v[i];
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {                     // zeros behind the rank
            const uint32_t e = i * Threads + thread;
            if (e % (4 * S) >= per) *reinterpret_cast<u32x4 *>(columns + e / (4 * S) * kColumn<S> + e % (4 * S) * 16) = u32x4{0, 0, 0, 0};
        }
    }
};

// The columns [from, to) that row y of the grid has, of a slice that ends at `end`; `width` at a time.
struct Range {
    int slice = 0;
    int32_t from, to, end;
    __device__ __forceinline__ Range(const Expansion &p, int32_t width)
    {
        const int32_t chunk = blockIdx.y;
        while (slice + 1 < p.slices && chunk >= p.cut.first_chunk[slice + 1]) ++slice;
        end = p.cut.first_column[slice + 1];
        from = p.cut.first_column[slice] + (chunk - p.cut.first_chunk[slice]) * p.chunks * width;
        to = from + p.chunks * width < end ? from + p.chunks * width : end;
    }
};

// Items of sixteen rows: every wave has columns of its own, 64 at a time, and waits for no other.  64 rows of 32 adapters, rank 16, 8192 columns: 7.4
// us, two thirds of it the launch and three latencies, one after the other: the item, what it names, the result.  kRows: an item for every row, some of none.
constexpr int kFewWaves = 4;

template <int S, bool kRows, bool kNarrow, bool kStreams>
__global__ __launch_bounds__(64 * kFewWaves) void expand_few_kernel(const Expansion p)
{
    static_assert(16 * kResult <= 64 * kColumn<S>, "results have the columns' place");
    __shared__ __align__(16) uint8_t lds[kFewWaves][64 * kColumn<S>];
    const int32_t at = kRows ? (int32_t)blockIdx.x : item_of(blockIdx.x, gridDim.x, p.together);
    SixteenRows<S, kNarrow, kStreams> sixteen(p, p.order + (int64_t)at * 16);
    const Item item = p.items[at];
    if (item.count == 0) return;
    const int wave = threadIdx.x >> 6;
    const Range range(p, 64 * kFewWaves);
    const int32_t from = range.from + wave * 64;
    if (from >= range.to) return;
    const uint8_t *const adapter = reinterpret_cast<const uint8_t *>(p.b + (int64_t)item.adapter * p.N * p.rank);
    const uint32_t per = (uint32_t)p.rank / 8;
    Columns<S, 64> columns;
    columns.load(adapter, per, from, range.end);
    sixteen.take(p, item.count);
    typename SixteenRows<S, kNarrow, kStreams>::Before before[2];
    sixteen.load(before[0], from);
    sixteen.join(p, range.slice, p.factors[item.adapter]);
    // Two turns a round, so that what a turn asks for has registers of its own; it is asked for before the turn's own stores, which a wait for it would
    // have to wait for too.
    auto turn = [&](int32_t n0, int which) {
        const int32_t n1 = n0 + 64 * kFewWaves < range.to ? n0 + 64 * kFewWaves : n0;
        columns.put(lds[wave], per);
        in_wave_order();
        columns.load(adapter, per, n1, range.end);
        sixteen.load(before[which ^ 1], n1);
        v4f sum[4] = {};
        sixteen.multiply_columns(lds[wave], sum);
        in_wave_order();
        sixteen.store(sum, before[which], lds[wave], n0, range.end);
    };
    for (int32_t n0 = from; n0 < range.to; n0 += 2 * 64 * kFewWaves) {
        turn(n0, 0);
        if (n0 + 64 * kFewWaves < range.to) turn(n0 + 64 * kFewWaves, 1);
    }
}

// Items of 64 rows: four waves of sixteen share 64 columns at a time, in two places in turn, so that B is read once for all of them (every sixteen rows
// reading it for themselves were bound by that: 4096 rows, rank 64, 5376 columns 28 us).  What bounds it now is latency between its barriers, two
// workgroups a CU: 22 us for the 88 MB of out, 4.0 TB/s.
template <int S, bool kStreams>
__global__ __launch_bounds__(256) void expand_many_kernel(const Expansion p)
{
    __shared__ __align__(16) uint8_t lds[2][64 * kColumn<S>], results[4][16 * kResult];
    const int32_t at = item_of(blockIdx.x, gridDim.x, p.together);
    const int wave = threadIdx.x >> 6;
    SixteenRows<S, false, kStreams> sixteen(p, p.order + (int64_t)at * 64 + wave * 16);
    const Item item = p.items[at];
    if (item.count == 0) return;
    const Range range(p, 64);
    const int32_t count = item.count - wave * 16;
    if (count <= 0) sixteen = SixteenRows<S, false, kStreams>(p, p.order + (int64_t)at * 64);
    const uint8_t *const adapter = reinterpret_cast<const uint8_t *>(p.b + (int64_t)item.adapter * p.N * p.rank);
    const uint32_t per = (uint32_t)p.rank / 8;
    Columns<S, 256> columns;
    columns.load(adapter, per, range.from, range.end);
    sixteen.take(p, count);
    typename SixteenRows<S, false, kStreams>::Before before[2];
    sixteen.load(before[0], range.from);
    sixteen.join(p, range.slice, p.factors[item.adapter]);
    auto turn = [&](int32_t n0, int which) {
        const int32_t n1 = n0 + 64 < range.to ? n0 + 64 : n0;
        columns.put(lds[which], per);
        __syncthreads();                        // the other place is written again only after the next
        columns.load(adapter, per, n1, range.end);
        sixteen.load(before[which ^ 1], n1);
        if (count > 0) {
            v4f sum[4] = {};
            sixteen.multiply_columns(lds[which], sum);
            sixteen.store(sum, before[which], results[wave], n0, range.end);
        }
    };
    for (int32_t n0 = range.from; n0 < range.to; n0 += 128) {
        turn(n0, 0);
        if (n0 + 64 < range.to) turn(n0 + 64, 1);
    }
}

}  // namespace adapters
}  // namespace equarx
