// Device code of low-rank adapters of many requests: rows brought together by adapter, t = A x, and out += f B t.
#pragma once

#include "equarx.h"
#include "equarx_rows.hpp"

namespace equarx {
namespace adapters {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMostSlices = EQUARX_ADAPTERS_MAX_SLICES, kMostAdapters = EQUARX_ADAPTERS_MAX;

// Rows of one adapter that are taken together: `count` of them from order[first] on.
struct Item {
    int32_t adapter, first, count, unused;
};

// ---------------------------------------------------------------- rows by adapter
// One workgroup counts, lays out and places.  Which of an adapter's rows comes first is left to the atomics: a row's results are its
// own column of the products below and do not depend on its place.

__global__ __launch_bounds__(1024) void group_kernel(Global<const int32_t> ids, int32_t M, int32_t adapters, int32_t tile, Global<int32_t> order,
                                                     Global<Item> items, Global<int32_t> item_count)
{
    __shared__ int32_t at[kMostAdapters];
    __shared__ int32_t part_rows[16], part_items[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int a = threadIdx.x; a < adapters; a += 1024) at[a] = 0;
    __syncthreads();
    for (int32_t m = threadIdx.x; m < M; m += 1024) {
        const int32_t a = ids[m];
        if (a >= 0 && a < adapters) atomicAdd(&at[a], 1);
    }
    __syncthreads();
    int32_t rows = 0, done = 0;
    for (int a0 = 0; a0 < adapters; a0 += 1024) {
        const int a = a0 + (int)threadIdx.x;
        const int32_t n = a < adapters ? at[a] : 0, pieces = (n + tile - 1) / tile;
        int32_t r = n, p = pieces;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t ro = __shfl_up(r, d), po = __shfl_up(p, d);
            if (lane >= d) {
                r += ro;
                p += po;
            }
        }
        __syncthreads();
        if (lane == 63) {
            part_rows[wave] = r;
            part_items[wave] = p;
        }
        __syncthreads();
        int32_t row = rows + r - n, item = done + p - pieces;
        for (int i = 0; i < 16; ++i) {
            if (i < wave) {
                row += part_rows[i];
                item += part_items[i];
            }
            rows += part_rows[i];
            done += part_items[i];
        }
        if (a < adapters) at[a] = row;
        for (int32_t i = 0; i < pieces; ++i)
            items[item + i] = Item{a, row + i * tile, n - i * tile < tile ? n - i * tile : tile, 0};
    }
    if (threadIdx.x == 0) item_count[0] = done;
    __syncthreads();
    for (int32_t m = threadIdx.x; m < M; m += 1024) {
        const int32_t a = ids[m];
        if (a >= 0 && a < adapters) order[atomicAdd(&at[a], 1)] = m;
    }
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
// A workgroup has an item's rows, 64 rows of A and a piece of k; its four waves take 64 of k in turn.  Partial sums of the pieces go
// to t [split][M][R].

constexpr int kRankTile = 64, kStep = 64, kWaveSteps = 4 * kStep;

template <int RT>
__global__ __launch_bounds__(256) void shrink_kernel(Global<const uint16_t> x, int64_t x_stride, Global<const uint16_t> a, Global<float> t,
                                                     int32_t M, int32_t K, int32_t R, int32_t piece, Global<const int32_t> order,
                                                     Global<const Item> items, Global<const int32_t> item_count)
{
    constexpr int T = 16 * RT;
    __shared__ __align__(16) float sums[4][T][kRankTile];
    if ((int32_t)blockIdx.x >= item_count[0]) return;
    const Item item = items[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int32_t r0 = blockIdx.y * kRankTile, k_from = blockIdx.z * piece, k_to = k_from + piece < K ? k_from + piece : K;
    const uint16_t *xr[RT], *ar[4];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int32_t at = i * 16 + l < item.count ? i * 16 + l : item.count - 1;
        xr[i] = x + order[item.first + at] * x_stride;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t r = r0 + i * 16 + l < R ? r0 + i * 16 + l : R - 1;
        ar[i] = a + ((int64_t)item.adapter * R + r) * K;
    }
    v4f sum[RT][4] = {};
    for (int32_t k0 = k_from + wave * kStep; k0 < k_to; k0 += kWaveSteps) {
        const int32_t k = k0 + g * 16;
        u32x4 xv[RT][2], av[4][2];
        if (k0 + kStep <= k_to) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < RT; ++i) xv[i][j] = load8(xr[i] + k + 8 * j);
#pragma unroll
                for (int i = 0; i < 4; ++i) av[i][j] = load8(ar[i] + k + 8 * j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < RT; ++i) xv[i][j] = load_row8(xr[i], k + 8 * j, k_to);
#pragma unroll
                for (int i = 0; i < 4; ++i) av[i][j] = load_row8(ar[i], k + 8 * j, k_to);
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[i][q] = multiply(av[q][j], xv[i][j], sum[i][q]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<v4f *>(&sums[wave][i * 16 + l][q * 16 + g * 4]) = sum[i][q];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < T * kRankTile / 4; i += 256) {
        const int row = i / (kRankTile / 4), r = i % (kRankTile / 4) * 4;
        if (row >= item.count || r0 + r >= R) continue;             // R is a multiple of 8
        v4f s = *reinterpret_cast<const v4f *>(&sums[0][row][r]);
#pragma unroll
        for (int w = 1; w < 4; ++w) s += *reinterpret_cast<const v4f *>(&sums[w][row][r]);
        *reinterpret_cast<v4f *>(t + ((int64_t)blockIdx.z * M + order[item.first + row]) * R + r0 + r) = s;
    }
}

// ---------------------------------------------------------------- out += f B t
// A workgroup has an item's rows and 256 columns of a slice, a wave 64 of them.  t, joined from its partial sums, is taken as two bf16, both halves
// side by side along the product's k: B's rows come round again for the second.  Tile i of a wave's four has of every sixteen
// columns the four from 4 i on, so that a lane ends with sixteen consecutive outputs of a row.

struct Slices {
    int32_t first_column[kMostSlices + 1], first_chunk[kMostSlices + 1];     // of the slices there are; the end after them
};

constexpr int kChunk = 256;                 // columns of a workgroup
constexpr int kMostSteps = 2 * EQUARX_ADAPTERS_MAX_RANK / 32;

template <int RT>
__global__ __launch_bounds__(256) void expand_kernel(Global<uint16_t> out, int64_t out_stride, Global<const uint16_t> b,
                                                     Global<const float> factors, Global<const float> t, int32_t M, int32_t N, int32_t rank,
                                                     int32_t slices, int32_t splits, Global<const int32_t> order, Global<const Item> items,
                                                     Global<const int32_t> item_count, const Slices cut)
{
    constexpr int T = 16 * RT;
    __shared__ __align__(16) uint8_t lds[T * (kMostSteps * 64 + 16)];       // rows of 2 * rank bf16, padded
    if ((int32_t)blockIdx.x >= item_count[0]) return;
    const Item item = items[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int32_t R = slices * rank, steps = (2 * rank + 31) / 32, pitch = steps * 64 + 16;
    const int32_t chunk = blockIdx.y;
    int s = 0;
    while (s + 1 < slices && chunk >= cut.first_chunk[s + 1]) ++s;
    const float factor = factors[item.adapter];
    const int32_t per_row = steps * 16;                         // pairs of rank entries, the padding among them
    for (int32_t i = threadIdx.x; i < T * per_row; i += 256) {
        const int32_t j = i % per_row * 2, row = i / per_row;
        uint32_t pair = 0;
        if (row < item.count && j < 2 * rank) {
            const int32_t k = j < rank ? j : j - rank;
            const float *p = t + (int64_t)order[item.first + row] * R + s * rank + k;
            float v[2] = {0, 0};
            for (int32_t q = 0; q < splits; ++q) {
                v[0] += p[(int64_t)q * M * R];
                v[1] += p[(int64_t)q * M * R + 1];
            }
            v[0] *= factor;
            v[1] *= factor;
            pair = narrow_bf16x2(v[0], v[1]);
            if (j >= rank) pair = narrow_bf16x2(v[0] - __uint_as_float(pair << 16), v[1] - __uint_as_float(pair & 0xffff0000u));
        }
        *reinterpret_cast<uint32_t *>(lds + row * pitch + j * 2) = pair;
    }
    __syncthreads();
    const int32_t n0 = cut.first_column[s] + (chunk - cut.first_chunk[s]) * kChunk + wave * 64, n_end = cut.first_column[s + 1];
    if (n0 >= n_end) return;
    const uint16_t *br[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t n = n0 + (l / 4) * 16 + i * 4 + l % 4;
        br[i] = b + ((int64_t)item.adapter * N + (n < n_end ? n : n_end - 1)) * rank;
    }
    v4f sum[RT][4] = {};
    for (int32_t step = 0; step < steps; ++step) {
        const int32_t j = step * 32 + g * 8;
        u32x4 bv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bv[i] = j < 2 * rank ? load8(br[i] + (j < rank ? j : j - rank)) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const u32x4 tv = *reinterpret_cast<const u32x4 *>(lds + (r * 16 + l) * pitch + j * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[r][i] = multiply(bv[i], tv, sum[r][i]);
        }
    }
    const int32_t n = n0 + g * 16;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (r * 16 + l >= item.count) continue;
        uint16_t *const row = out + order[item.first + r * 16 + l] * out_stride;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (n + half * 8 >= n_end) continue;
            float f[8];
            widen_bf16x8(load_row8(row, n + half * 8, n_end), f);
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v4f d = sum[r][half * 2 + i / 2];
                v[i] = narrow_bf16x2(f[2 * i] + d[i % 2 * 2], f[2 * i + 1] + d[i % 2 * 2 + 1]);
            }
            store_row8(row, n + half * 8, n_end, v);
        }
    }
}

}  // namespace adapters
}  // namespace equarx
