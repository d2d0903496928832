// Device code of the int8 key/value cache: writing tokens, reading sequences back, and attention.
#pragma once

#include "equarx_device.hpp"

namespace equarx {
namespace cache {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The pool as the kernels see it.
struct Pool {
    int8_t *kc;
    float *ks;
    int8_t *vc;
    float *vs;
    int64_t pages;
    int32_t heads, page;
    int32_t page_shift;         // log2(page), or -1

    // index of (page p, head h): the unit that codes (page * dim) and scales (blocks * page) are counted in
    __device__ __forceinline__ int64_t place(int64_t p, int h) const { return p * heads + h; }
};

// Sequences of a call.
struct Sequences {
    const int32_t *table;
    const int32_t *lengths;
    int64_t width;

    __device__ __forceinline__ int64_t length(int b, int page) const
    {
        const int64_t n = lengths[b], most = width * page;
        return n < 0 ? 0 : n < most ? n : most;
    }
};

__device__ __forceinline__ int page_of(const Pool &pool, int64_t t)
{
    return pool.page_shift >= 0 ? (int)(t >> pool.page_shift) : (int)((uint32_t)t / (uint32_t)pool.page);
}

// 4x4 bytes, rows in and columns out.
__device__ __forceinline__ u32x4 transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab_lo = __builtin_amdgcn_perm(b, a, 0x05010400u), ab_hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd_lo = __builtin_amdgcn_perm(d, c, 0x05010400u), cd_hi = __builtin_amdgcn_perm(d, c, 0x07030602u);
    return u32x4{__builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100u), __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302u),
                 __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100u), __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302u)};
}

// ---------------------------------------------------------------- writing
// A lane has eight elements of four consecutive tokens of the call, dim / 8 lanes a head.  Keys are written eight bytes at a
// time; values four tokens together where the four lie in one group of sixteen slots from a multiple of four on, and byte
// by byte where they do not.

// Q_B of eight bf16 numbers, a block being the 8 * G elements of G lanes; a NaN scale where the block is not finite.
template <int G>
__device__ __forceinline__ u32x2 quantize_finite(const u32x4 &x, float &scale)
{
    float t[8];
    widen_bf16x8(x, t);
    const u32x2 codes = quantize_lane<G>(t, scale);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = umax(top, __float_as_uint(t[i]) & 0x7fffffffu);
    if (group_max_bits<G>(top) >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);
    return codes;
}

template <int D, int B>
__global__ __launch_bounds__(256) void write_kernel(Global<const uint16_t> k, Global<const uint16_t> v,
                                                    Global<const int64_t> slots, int64_t k_row, int64_t v_row,
                                                    int32_t tokens, int64_t k_head, int64_t v_head, const Pool pool)
{
    constexpr int kLanes = D / 8, kBlocks = D / B, G = B / 8;
    const int h = blockIdx.y;
    const int t0 = (blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes) * 4;
    const int d = threadIdx.x % kLanes * 8;
    const int64_t space = pool.pages * pool.page;
    u32x4 kx[4], vx[4];
    int64_t slot[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = t0 + i < tokens ? t0 + i : tokens - 1;
        slot[i] = t0 + i < tokens ? slots[t] : -1;
        if (slot[i] >= space) slot[i] = -1;
        kx[i] = *reinterpret_cast<const u32x4 *>(k + t * k_row + h * k_head + d);
        vx[i] = *reinterpret_cast<const u32x4 *>(v + t * v_row + h * v_head + d);
    }
    loads_first();
    u32x2 vw[4];
    int64_t at[4];
    int in_page[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float ks, vs;
        const u32x2 kw = quantize_finite<G>(kx[i], ks);
        vw[i] = quantize_finite<G>(vx[i], vs);
        const int64_t p = slot[i] < 0 ? 0 : pool.page_shift >= 0 ? slot[i] >> pool.page_shift : slot[i] / pool.page;
        at[i] = pool.place(p, h);
        in_page[i] = (int)(slot[i] - p * pool.page);
        if (slot[i] >= 0) {
            *reinterpret_cast<u32x2 *>(pool.kc + at[i] * pool.page * D + in_page[i] * D + d) = kw;
            if (d % B == 0) {
                const int64_t s = at[i] * pool.page * kBlocks + d / B * pool.page + in_page[i];
                pool.ks[s] = ks;
                pool.vs[s] = vs;
            }
        }
    }
    const bool together = slot[0] >= 0 && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 &&
                          slot[3] == slot[0] + 3;
    if (together) {
        int8_t *const to = pool.vc + at[0] * pool.page * D + (int64_t)(in_page[0] & ~15) * D + d * 16 + (in_page[0] & 15);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 w = transpose4(vw[0][j], vw[1][j], vw[2][j], vw[3][j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t *>(to + (4 * j + i) * 16) = w[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (slot[i] < 0) continue;
        int8_t *const to = pool.vc + at[i] * pool.page * D + (int64_t)(in_page[i] & ~15) * D + d * 16 + (in_page[i] & 15);
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j * 16] = (int8_t)(vw[i][j / 4] >> (8 * (j % 4)));
    }
}

// ---------------------------------------------------------------- reading back
// A lane has eight elements of four tokens from a multiple of four on, dim / 8 lanes a head.

__device__ __forceinline__ u32x4 read_back(const u32x2 &codes, float scale)
{
    float f[8];
    widen_i8x8(codes, f);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = narrow_bf16x2(f[2 * i] * scale, f[2 * i + 1] * scale);
    return w;
}

template <int D, int B>
__global__ __launch_bounds__(256) void read_kernel(Global<uint16_t> k_out, Global<uint16_t> v_out, Global<const int32_t> starts,
                                                   int64_t rows, const Sequences seqs, const Pool pool)
{
    constexpr int kLanes = D / 8, kBlocks = D / B, kTokens = 256 / kLanes * 4;
    const int b = blockIdx.z, h = blockIdx.y;
    const int d = threadIdx.x % kLanes * 8;
    const int64_t length = seqs.length(b, pool.page), start = starts[b];
    for (int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes * 4; t < length; t += (int64_t)gridDim.x * kTokens) {
        const int p = page_of(pool, t);
        const int i0 = (int)(t - (int64_t)p * pool.page);
        const int64_t id = seqs.table[b * seqs.width + p];
        const bool there = id >= 0 && id < pool.pages;
        const int64_t at = pool.place(there ? id : 0, h) * pool.page;
        u32x2 kw[4], vw[4];
        float ks[4], vs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) kw[i] = *reinterpret_cast<const u32x2 *>(pool.kc + (at + i0 + i) * D + d);
        uint32_t quad[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            quad[j] = *reinterpret_cast<const uint32_t *>(pool.vc + (at + (i0 & ~15)) * D + (d + j) * 16 + (i0 & 15));
        const int64_t s = at * kBlocks + d / B * pool.page + i0;
        const v4f ks4 = *reinterpret_cast<const v4f *>(pool.ks + s), vs4 = *reinterpret_cast<const v4f *>(pool.vs + s);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 w = transpose4(quad[4 * j], quad[4 * j + 1], quad[4 * j + 2], quad[4 * j + 3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) vw[i][j] = w[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ks[i] = there ? ks4[i] : 0.0f;
            vs[i] = there ? vs4[i] : 0.0f;
            const int64_t row = start + t + i;
            if (t + i < length && row >= 0 && row < rows) {
                const int64_t o = (row * pool.heads + h) * D + d;
                *reinterpret_cast<u32x4 *>(k_out + o) = read_back(kw[i], ks[i]);
                *reinterpret_cast<u32x4 *>(v_out + o) = read_back(vw[i], vs[i]);
            }
        }
    }
}

// ---------------------------------------------------------------- attention
// A wave has R * 16 query rows of one key head -- (query, member of the head's group of query heads) pairs, the members of a
// query next to each other -- and walks over tokens, 64 at a time, everything in registers:
//
//   scores   S^T = K Q^T with 16x16x32 instructions, four times 16 tokens by 16 rows.  The tokens of an instruction's rows are
//            chosen so that its result leaves lane (row c = l % 16, quarter g = l / 16) with the tokens 16 g + 4 s + i, s and i
//            from 0 to 3: after the four, the tokens 16 g .. 16 g + 15 in order.
//   sums     O^T += V^T P^T takes a lane's P as it is: quarter g has 8 consecutive tokens of its 16 per instruction, and the 16
//            codes of one element of v for those tokens are 16 consecutive bytes of the cache.
// A code is exact in bf16; scales join in fp32, the keys' on the scores, the values' on the probabilities before these are
// rounded to bf16 (up to 2^-8 of each summand, as any attention that feeds matrix instructions has it).  Running maximum and sum per
// row; the sum stays split over the quarters until the end.

struct AttentionCall {
    const uint16_t *q;
    int64_t q_row, q_head;
    const int32_t *q_starts;
    uint16_t *out;
    float *lse;
    float *part;                // [splits][q_rows][q_heads][D], then the statistics, 2 each
    int64_t q_rows;
    int32_t q_heads, group;
    float scale;                // times log2(e)
    int32_t causal, window;
    int32_t chunk;              // tokens of a split, a multiple of 64
    int32_t splits;
};

__device__ __forceinline__ int64_t within(int64_t v, int64_t most) { return v < 0 ? 0 : v < most ? v : most; }

// The factor that ends a row: 1 / its sum, 0 for a row that saw nothing (whose sum is 0, where any token seen adds up to 1
// at least, or to NaN), and its log sum of exponentials.
__device__ __forceinline__ float ends_with(float total) { return total == 0.0f ? 0.0f : 1.0f / total; }
__device__ __forceinline__ float log_sum(float top, float total)
{
    return total == 0.0f ? -__builtin_inff() : (top + __builtin_log2f(total)) * 0.69314718056f;
}

__device__ __forceinline__ float quarters_max(float v)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float a = __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(a), false, false);
    return __builtin_fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

__device__ __forceinline__ float quarters_sum(float v)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float a = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(a), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

__device__ __forceinline__ bf16x8 widen_codes(uint32_t a, uint32_t b)
{
    float f[8];
    widen_i8x8(u32x2{a, b}, f);
    const u32x4 w = {narrow_bf16x2(f[0], f[1]), narrow_bf16x2(f[2], f[3]), narrow_bf16x2(f[4], f[5]), narrow_bf16x2(f[6], f[7])};
    return __builtin_bit_cast(bf16x8, w);
}

// What a wave has of 64 tokens.
template <int D, int NB>
struct Tile {
    u32x4 k[4][D / 64], v[D / 16];
    v4f ks[NB][4], vs[NB][4];

    // `k_at`, `v_at`: of this lane's K token group and of its V token group, the pool's first element
    __device__ __forceinline__ void load(const Pool &pool, int64_t k_at, int64_t v_at, int k_in, int v_in, int lane)
    {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int8_t *const row = pool.kc + (k_at * pool.page + k_in + 4 * s + (r & 3)) * D + g * 16;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) k[s][j] = *reinterpret_cast<const u32x4 *>(row + 64 * j);
        }
        const int64_t scales = v_at * pool.page * NB + v_in;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                ks[n][s] = *reinterpret_cast<const v4f *>(pool.ks + scales + n * pool.page + 4 * s);
                vs[n][s] = *reinterpret_cast<const v4f *>(pool.vs + scales + n * pool.page + 4 * s);
            }
        const int8_t *const values = pool.vc + (v_at * pool.page + v_in) * D + r * 16;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) v[t] = *reinterpret_cast<const u32x4 *>(values + t * 256);
    }
};

// Waves of a workgroup: on the same rows and different tokens (kTokens), their results joined at the end, or on
// different rows.
template <int D, int NB, int R, bool kTokens>
__global__ __launch_bounds__(256) void attention_kernel(const AttentionCall call, const Sequences seqs, const Pool pool)
{
    constexpr int W = 4;
    constexpr float kNone = -__builtin_inff();
    __shared__ float joined[kTokens ? W : 1][kTokens ? R * 16 : 1][D + 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int b = blockIdx.z, h = blockIdx.y % pool.heads, split = blockIdx.y / pool.heads;
    const int64_t q0 = within(call.q_starts[b], call.q_rows);
    const int queries = (int)(within(call.q_starts[b + 1], call.q_rows) - q0);
    const int64_t length = seqs.length(b, pool.page);
    // this split's tokens: whole tiles; a sequence longer than the host knew has longer splits
    int64_t chunk = call.chunk;
    if (chunk * call.splits < length) chunk = (length + call.splits - 1) / call.splits + 63 & ~(int64_t)63;

    const int64_t rows = (int64_t)queries * call.group;
    constexpr int kRows = (kTokens ? 1 : W) * R * 16;
    for (int64_t tile_row = (int64_t)blockIdx.x * kRows; tile_row < rows; tile_row += (int64_t)gridDim.x * kRows) {
        const int64_t row0 = tile_row + (kTokens ? 0 : wave * R * 16);
        // the rows of this lane: their query's position, their q in registers
        int64_t place[R];
        int64_t q_row[R];
        int member[R];
        bf16x8 q[R][D / 32];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            const int64_t row = row0 + n * 16 + r < rows ? row0 + n * 16 + r : rows - 1;
            const int i = (int)(row / call.group);
            member[n] = h * call.group + (int)(row - (int64_t)i * call.group);
            q_row[n] = q0 + i;
            place[n] = length - queries + i;
            const uint16_t *const from = call.q + q_row[n] * call.q_row + member[n] * call.q_head + g * 16;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                q[n][j] = *reinterpret_cast<const bf16x8 *>(from + (j / 2) * 64 + (j % 2) * 8);
        }
        // what any row of the workgroup sees
        int64_t first = split * chunk, last = first + chunk < length ? first + chunk : length;
        const int64_t tile_last = tile_row + kRows < rows ? tile_row + kRows - 1 : rows - 1;
        const int64_t low = length - queries + tile_row / call.group, high = length - queries + tile_last / call.group;
        if (call.causal) {
            if (high + 1 < last) last = high + 1;
            if (call.window && low - call.window + 1 > first) first = (low - call.window + 1) & ~(int64_t)63;
        }

        v4f o[R][D / 16];
        float top[R], total[R];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            top[n] = kNone;
            total[n] = 0.0f;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) o[n][t] = v4f{0, 0, 0, 0};
        }

        for (int64_t t0 = first + (kTokens ? wave * 64 : 0); t0 < last; t0 += (kTokens ? W : 1) * 64) {
            Tile<D, NB> tile;
            const int64_t k_t = t0 + 16 * (r >> 2), v_t = t0 + 16 * g;
            const int k_p = page_of(pool, k_t), v_p = page_of(pool, v_t);
            int64_t k_id = k_p < seqs.width ? seqs.table[b * seqs.width + k_p] : -1;
            int64_t v_id = v_p < seqs.width ? seqs.table[b * seqs.width + v_p] : -1;
            const bool there = v_id >= 0 && v_id < pool.pages;
            if (k_id < 0 || k_id >= pool.pages) k_id = 0;
            if (!there) v_id = 0;
            tile.load(pool, pool.place(k_id, h), pool.place(v_id, h), (int)(k_t - (int64_t)k_p * pool.page),
                      (int)(v_t - (int64_t)v_p * pool.page), lane);

            v4f score[R][4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                v4f dot[R][NB];
#pragma unroll
                for (int n = 0; n < R; ++n)
#pragma unroll
                    for (int m = 0; m < NB; ++m) dot[n][m] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const bf16x8 a0 = widen_codes(tile.k[s][j][0], tile.k[s][j][1]);
                    const bf16x8 a1 = widen_codes(tile.k[s][j][2], tile.k[s][j][3]);
                    constexpr int kPer = D / 64 / NB;
#pragma unroll
                    for (int n = 0; n < R; ++n) {
                        v4f &to = dot[n][j / kPer];
                        to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, q[n][2 * j], to, 0, 0, 0);
                        to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, q[n][2 * j + 1], to, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int n = 0; n < R; ++n) {
                    score[n][s] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int m = 0; m < NB; ++m)
#pragma unroll
                        for (int i = 0; i < 4; ++i) score[n][s][i] = __builtin_fmaf(dot[n][m][i], tile.ks[m][s][i], score[n][s][i]);
                }
            }
            bf16x8 p[R][NB][2];
#pragma unroll
            for (int n = 0; n < R; ++n) {
                uint32_t seen = 0;          // a bit per token of this lane
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t t = v_t + 4 * s + i;
                        const bool sees = there && t < length && (!call.causal || (t <= place[n] && (!call.window || t > place[n] - call.window)));
                        seen |= (uint32_t)sees << (4 * s + i);
                        score[n][s][i] = sees ? score[n][s][i] * call.scale : kNone;
                    }
                float most = kNone;
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most = __builtin_fmaxf(most, score[n][s][i]);
                const float now = __builtin_fmaxf(top[n], quarters_max(most));
                const float base = now == kNone ? 0.0f : now;
                const float fade = __builtin_amdgcn_exp2f(top[n] - base);
                top[n] = now;
                float e[16];
                float sum = 0.0f;
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e[4 * s + i] = __builtin_amdgcn_exp2f(score[n][s][i] - base);
                        sum += e[4 * s + i];
                    }
                total[n] = total[n] * fade + sum;
#pragma unroll
                for (int t = 0; t < D / 16; ++t) o[n][t] *= fade;
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    u32x4 w[2];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float lo = seen >> (2 * j) & 1 ? e[2 * j] * tile.vs[m][j / 2][2 * (j % 2)] : 0.0f;
                        const float hi = seen >> (2 * j + 1) & 1 ? e[2 * j + 1] * tile.vs[m][j / 2][2 * (j % 2) + 1] : 0.0f;
                        w[j / 4][j % 4] = narrow_bf16x2(lo, hi);
                    }
                    p[n][m][0] = __builtin_bit_cast(bf16x8, w[0]);
                    p[n][m][1] = __builtin_bit_cast(bf16x8, w[1]);
                }
            }
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                const bf16x8 a0 = widen_codes(tile.v[t][0], tile.v[t][1]), a1 = widen_codes(tile.v[t][2], tile.v[t][3]);
                constexpr int kPer = D / 16 / NB;
#pragma unroll
                for (int n = 0; n < R; ++n) {
                    o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, p[n][t / kPer][0], o[n][t], 0, 0, 0);
                    o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, p[n][t / kPer][1], o[n][t], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < R; ++n) total[n] = quarters_sum(total[n]);

        if constexpr (kTokens) {            // join the four waves
            __syncthreads();                // the last rows' results have been read
#pragma unroll
            for (int n = 0; n < R; ++n) {
#pragma unroll
                for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(&joined[wave][n * 16 + r][t * 16 + 4 * g]) = o[n][t];
                if (g == 0) {
                    joined[wave][n * 16 + r][D] = top[n];
                    joined[wave][n * 16 + r][D + 1] = total[n];
                }
            }
            __syncthreads();
            constexpr int kLanes = D / 4;   // of a row
            for (int i = threadIdx.x; i < R * 16 * kLanes; i += 256) {
                const int row = i / kLanes, d = i % kLanes * 4;
                if (row0 + row >= rows) continue;
                float now = kNone;
#pragma unroll
                for (int w = 0; w < W; ++w) now = __builtin_fmaxf(now, joined[w][row][D]);
                const float base = now == kNone ? 0.0f : now;
                float sum = 0.0f;
                v4f acc = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float fade = __builtin_amdgcn_exp2f(joined[w][row][D] - base);
                    sum += joined[w][row][D + 1] * fade;
                    acc += *reinterpret_cast<const v4f *>(&joined[w][row][d]) * fade;
                }
                const int64_t qi = (row0 + row) / call.group;
                const int64_t place_out = (q0 + qi) * call.q_heads + h * call.group + (row0 + row - qi * call.group);
                if (call.splits > 1) {
                    const int64_t at = split * call.q_rows * call.q_heads + place_out;
                    *reinterpret_cast<v4f *>(call.part + at * D + d) = acc;
                    if (d == 0) {
                        float *const stats = call.part + call.splits * call.q_rows * call.q_heads * D + at * 2;
                        stats[0] = now;
                        stats[1] = sum;
                    }
                } else {
                    const float inverse = ends_with(sum);
                    const u32x2 w = {narrow_bf16x2(acc[0] * inverse, acc[1] * inverse), narrow_bf16x2(acc[2] * inverse, acc[3] * inverse)};
                    *reinterpret_cast<u32x2 *>(call.out + place_out * D + d) = w;
                    if (call.lse && d == 0) call.lse[place_out] = log_sum(now, sum);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < R; ++n) {
                if (row0 + n * 16 + r >= rows) continue;
                const int64_t place_out = q_row[n] * call.q_heads + member[n];
                if (call.splits > 1) {
                    const int64_t at = split * call.q_rows * call.q_heads + place_out;
#pragma unroll
                    for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(call.part + at * D + t * 16 + 4 * g) = o[n][t];
                    if (g == 0) {
                        float *const stats = call.part + call.splits * call.q_rows * call.q_heads * D + at * 2;
                        stats[0] = top[n];
                        stats[1] = total[n];
                    }
                } else {
                    const float inverse = ends_with(total[n]);
#pragma unroll
                    for (int t = 0; t < D / 16; ++t) {
                        const u32x2 w = {narrow_bf16x2(o[n][t][0] * inverse, o[n][t][1] * inverse),
                                         narrow_bf16x2(o[n][t][2] * inverse, o[n][t][3] * inverse)};
                        *reinterpret_cast<u32x2 *>(call.out + place_out * D + t * 16 + 4 * g) = w;
                    }
                    if (call.lse && g == 0)
                        call.lse[place_out] = log_sum(top[n], total[n]);
                }
            }
        }
    }
}

// Joins the splits of every output row: D / 4 lanes a row.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(const AttentionCall call, int32_t sequences)
{
    constexpr int kLanes = D / 4;
    constexpr float kNone = -__builtin_inff();
    const int64_t all = call.q_rows * call.q_heads;
    const int64_t at = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
    const int d = threadIdx.x % kLanes * 4;
    if (at >= all) return;
    const int64_t row = at / call.q_heads;
    if (row < call.q_starts[0] || row >= call.q_starts[sequences]) return;      // a row of no sequence
    const float *const stats = call.part + call.splits * all * D;
    float now = kNone;
    for (int s = 0; s < call.splits; ++s) now = __builtin_fmaxf(now, stats[(s * all + at) * 2]);
    const float base = now == kNone ? 0.0f : now;
    float sum = 0.0f;
    v4f acc = {0, 0, 0, 0};
    for (int s = 0; s < call.splits; ++s) {
        const float fade = __builtin_amdgcn_exp2f(stats[(s * all + at) * 2] - base);
        sum += stats[(s * all + at) * 2 + 1] * fade;
        acc += *reinterpret_cast<const v4f *>(call.part + (s * all + at) * D + d) * fade;
    }
    const float inverse = ends_with(sum);
    const u32x2 w = {narrow_bf16x2(acc[0] * inverse, acc[1] * inverse), narrow_bf16x2(acc[2] * inverse, acc[3] * inverse)};
    *reinterpret_cast<u32x2 *>(call.out + at * D + d) = w;
    if (call.lse && d == 0) call.lse[at] = log_sum(now, sum);
}

}  // namespace cache
}  // namespace equarx
