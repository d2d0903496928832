// Device code of low-rank adapters of many requests: rows brought together by adapter, t = A x, and out += f B t.
#pragma once

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
        const uint64_t same = __ballot(left && a == __shfl(a, first));
        if (left && (same >> lane & 1)) {
            int32_t base = 0;
            if (lane == first) base = atomicAdd(&at[a], (int32_t)__popcll(same));
            found = __shfl(base, first) + (int32_t)__popcll(same & (((uint64_t)1 << lane) - 1));
            left = false;
        }
    }
    if (left) found = atomicAdd(&at[a], 1);
    return found;
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
        int32_t p = pieces;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t other = __shfl_up(p, d);
            if (lane >= d) p += other;
        }
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
    return places[lane % 16 < item.count ? lane % 16 : 0];      // its own wave's writes, in order
}

// ---------------------------------------------------------------- products of sixteen by sixteen
// v_mfma_f32_16x16x32_bf16: lane l has row l % 16 of the first operand and column l % 16 of the second, k = 8 (l / 16) + 0 .. 7 of both,
// and of the result column l % 16, rows 4 (l / 16) + 0 .. 3.  Rows of x are always the columns: a NaN or an infinity stays in its row.

__device__ __forceinline__ v4f multiply(const u32x4 &a, const u32x4 &b, const v4f &sum)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), sum, 0, 0, 0);
}

__device__ __forceinline__ u32x4 load8(const uint16_t *p) { return *reinterpret_cast<const u32x4_anywhere *>(p); }

// ---------------------------------------------------------------- t = A x
// A workgroup has an item's rows, 16 RT of them, 16 QT rows of A and a piece of k, of which its W waves take 64 in turn; their sums are
// added in order through LDS.  Sums of the pieces go to t [split][M][R].
// kFew: items are found here, and the first workgroup of each writes it down for the launch that follows.

constexpr int kStep = 64;

template <int RT, int QT, int W, bool kFew>
__global__ __launch_bounds__(64 * W) void shrink_kernel(Global<const uint16_t> x, int64_t x_stride, Global<const uint16_t> a, Global<float> t,
                                                        int32_t M, int32_t K, int32_t R, int32_t piece, Global<int32_t> order, Global<Item> items,
                                                        Global<const int32_t> ids, int32_t adapters)
{
    constexpr int T = 16 * RT, kPitch = QT * 16 + 4;
    constexpr int U = RT == 1 ? 2 : 1;                          // steps whose loads are asked for together
    __shared__ __align__(16) float sums[W][16][kPitch];
    __shared__ int32_t places[kFew ? W : 1][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    Item item;
    int32_t row[RT];
    if constexpr (kFew) {
        row[0] = find_item(ids, M, adapters, (int32_t)blockIdx.x, places[wave], item);
        if (blockIdx.y == 0 && blockIdx.z == 0 && wave == 0) {
            if (lane == 0) items[blockIdx.x] = item;
            if (lane < item.count) order[blockIdx.x * 16 + lane] = row[0];
        }
    } else {
        item = items[blockIdx.x];
#pragma unroll
        for (int i = 0; i < RT; ++i) row[i] = order[blockIdx.x * T + (i * 16 + l < item.count ? i * 16 + l : 0)];
    }
    if (item.count == 0) return;
    const int32_t r0 = blockIdx.y * (16 * QT), k_from = blockIdx.z * piece, k_to = k_from + piece < K ? k_from + piece : K;
    const uint16_t *xr[RT], *ar[QT];
#pragma unroll
    for (int i = 0; i < RT; ++i) xr[i] = x + row[i] * x_stride;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        const int32_t r = r0 + q * 16 + l < R ? r0 + q * 16 + l : R - 1;
        ar[q] = a + ((int64_t)item.adapter * R + r) * K;
    }
    struct Step {
        u32x4 x[RT][2], a[QT][2];
    };
    auto load = [&](Step &to, int32_t k0) {
        const int32_t k = k0 + g * 16;
        auto each = [&](auto get) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < RT; ++i) to.x[i][j] = get(xr[i], k + 8 * j);
#pragma unroll
                for (int q = 0; q < QT; ++q) to.a[q][j] = get(ar[q], k + 8 * j);
            }
        };
        if (k0 + kStep <= k_to) {
            each([](const uint16_t *p, int32_t at) { return load8(p + at); });
        } else if (k0 >= k_to) {
            each([](const uint16_t *, int32_t) { return u32x4{0, 0, 0, 0}; });
        } else if (K >= 8) {                                    // past the end zeros, in both
            each([&](const uint16_t *p, int32_t at) { return load_row8_back(p, at, K); });
        } else {
            each([&](const uint16_t *p, int32_t at) { return load_row8(p, at, K); });
        }
    };
    v4f sum[RT][QT] = {};
    auto add = [&](const Step &s) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
#pragma unroll
                for (int q = 0; q < QT; ++q) sum[i][q] = multiply(s.a[q][j], s.x[i][j], sum[i][q]);
            }
        }
    };
    constexpr int kNext = W * kStep;
    Step now[U];
    for (int32_t k0 = k_from + wave * kStep; k0 < k_to; k0 += U * kNext) {
#pragma unroll
        for (int u = 0; u < U; ++u) load(now[u], k0 + u * kNext);
#pragma unroll
        for (int u = 0; u < U; ++u) add(now[u]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int q = 0; q < QT; ++q) *reinterpret_cast<v4f *>(&sums[wave][l][q * 16 + g * 4]) = sum[i][q];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * QT * 4; e += 64 * W) {
            const int in = e / (QT * 4), r = e % (QT * 4) * 4;
            if (i * 16 + in >= item.count || r0 + r >= R) continue;             // R is a multiple of 8
            v4f s = *reinterpret_cast<const v4f *>(&sums[0][in][r]);
#pragma unroll
            for (int w = 1; w < W; ++w) s += *reinterpret_cast<const v4f *>(&sums[w][in][r]);
            const int32_t m = kFew ? places[0][in] : (int32_t)order[blockIdx.x * T + i * 16 + in];
            *reinterpret_cast<v4f *>(t + ((int64_t)blockIdx.z * M + m) * R + r0 + r) = s;
        }
    }
}

// ---------------------------------------------------------------- out += f B t
// A workgroup has an item's rows and chunks of 256 columns of a slice, a wave 64 of each.  t, joined from its partial sums, is taken as
// two bf16; one read of B's columns meets both halves of all rows, sixteen at a time.  Tile i of a wave's four has columns 32 (i / 2) + 8 g +
// 4 (i % 2) + 0 .. 3 for the four lane groups g, so that a lane ends with eight consecutive outputs, and the four groups with 64 bytes of a row.

struct Slices {
    int32_t first_column[kMostSlices + 1], first_chunk[kMostSlices + 1];     // of the slices there are; the end after them
};

constexpr int kChunk = 256;                 // columns that a workgroup takes at a time

// S: steps of 32 of the rank, at most.
template <int T, int S>
__global__ __launch_bounds__(256) void expand_kernel(Global<uint16_t> out, int64_t out_stride, Global<const uint16_t> b,
                                                     Global<const float> factors, Global<const float> t, int32_t M, int32_t N, int32_t rank,
                                                     int32_t slices, int32_t splits, int32_t chunks, Global<const int32_t> order,
                                                     Global<const Item> items, const Slices cut)
{
    constexpr int kPitch = S * 128 + 16;                        // bytes of a row of t: the first halves, the second, and a shift of banks
    __shared__ __align__(16) uint8_t lds[T * kPitch];
    const Item item = items[blockIdx.x];
    if (item.count == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int32_t R = slices * rank, chunk = blockIdx.y;
    int s = 0;
    while (s + 1 < slices && chunk >= cut.first_chunk[s + 1]) ++s;
    const int32_t n_end = cut.first_column[s + 1];
    const int32_t n_from = cut.first_column[s] + (chunk - cut.first_chunk[s]) * chunks * kChunk + wave * 64;
    const int32_t n_to = n_from + chunks * kChunk < n_end ? n_from + chunks * kChunk : n_end;
    const int32_t *const rows = order + (int64_t)blockIdx.x * T;
    const uint16_t *const mine = b + (int64_t)item.adapter * N * rank;
    struct Outputs {
        uint16_t *row;
        u32x4 v[2];
    };
    auto load_outputs = [&](Outputs &to, int32_t r, int32_t n0) {       // what is added to
        const bool real = r + l < item.count;
        to.row = real ? out + rows[r + l] * out_stride : nullptr;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int32_t n = n0 + half * 32 + g * 8;
            if (real && n < n_end) to.v[half] = load_row8(to.row, n, n_end);
        }
    };
    u32x4 entries[S][4];
    auto load_entries = [&](int32_t n0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t c = n0 + (i / 2) * 32 + (l / 4) * 8 + (i % 2) * 4 + l % 4;
            const uint16_t *const p = mine + (int64_t)(c < n_end ? c : n_end - 1) * rank;
#pragma unroll
            for (int q = 0; q < S; ++q) entries[q][i] = q * 32 + g * 8 < rank ? load8(p + q * 32 + g * 8) : u32x4{0, 0, 0, 0};
        }
    };
    Outputs now, next;
    if (n_from < n_to) {
        load_outputs(now, 0, n_from);
        load_entries(n_from);
    }
    const float factor = factors[item.adapter];
    // four entries of a row's rank at a time; zeros behind them
    for (int32_t e = threadIdx.x; e < T * S * 8; e += 256) {
        const int32_t row = e / (S * 8), k = e % (S * 8) * 4;
        v4f v = {0, 0, 0, 0};
        if (row < item.count && k < rank) {
            const float *const p = t + (int64_t)rows[row] * R + s * rank + k;
            for (int32_t q = 0; q < splits; ++q) v += *reinterpret_cast<const v4f *>(p + (int64_t)q * M * R);
            v *= factor;
        }
        const u32x2 high = {narrow_bf16x2(v[0], v[1]), narrow_bf16x2(v[2], v[3])};
        float h[4];
        widen_bf16x4(high, h);
        *reinterpret_cast<u32x2 *>(lds + row * kPitch + k * 2) = high;
        *reinterpret_cast<u32x2 *>(lds + row * kPitch + S * 64 + k * 2) =
            u32x2{narrow_bf16x2(v[0] - h[0], v[1] - h[1]), narrow_bf16x2(v[2] - h[2], v[3] - h[3])};
    }
    __syncthreads();
    for (int32_t n0 = n_from; n0 < n_to; n0 += kChunk) {
        if (n0 > n_from) load_entries(n0);
        for (int32_t r = 0; r < item.count; r += 16) {
            const bool last = r + 16 >= item.count;
            if (!last || n0 + kChunk < n_to) load_outputs(next, last ? 0 : r + 16, last ? n0 + kChunk : n0);
            v4f sum[4] = {};
            const uint8_t *const at = lds + (r + l) * kPitch + g * 16;
#pragma unroll
            for (int q = 0; q < S; ++q) {
                const u32x4 first = *reinterpret_cast<const u32x4 *>(at + q * 64), second = *reinterpret_cast<const u32x4 *>(at + S * 64 + q * 64);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = multiply(entries[q][i], second, multiply(entries[q][i], first, sum[i]));
            }
            if (now.row) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int32_t n = n0 + half * 32 + g * 8;
                    if (n >= n_end) continue;
                    float f[8];
                    widen_bf16x8(now.v[half], f);
                    u32x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const v4f d = sum[half * 2 + i / 2];
                        v[i] = narrow_bf16x2(f[2 * i] + d[i % 2 * 2], f[2 * i + 1] + d[i % 2 * 2 + 1]);
                    }
                    store_row8(now.row, n, n_end, v);
                }
            }
            now = next;
        }
    }
}

}  // namespace adapters
}  // namespace equarx
