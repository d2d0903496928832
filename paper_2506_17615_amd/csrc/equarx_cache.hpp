// Device code of the int8 key/value cache: writing tokens, reading sequences back, and attention.
#pragma once

#include <type_traits>
#include <utility>

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

// The longest sequence: a token's number, and what a loop adds to it, are 31 bits.
constexpr int64_t kMostTokens = ((int64_t)1 << 31) - 65536;

// Sequences of a call.
struct Sequences {
    const int32_t *table;
    const int32_t *lengths;
    int64_t width;

    __device__ __forceinline__ int length(int b, int page) const
    {
        const int64_t n = lengths[b], most = width * page < kMostTokens ? width * page : kMostTokens;
        return (int)(n < 0 ? 0 : n < most ? n : most);
    }
};

__device__ __forceinline__ int page_of(const Pool &pool, int t)
{
    return pool.page_shift >= 0 ? t >> pool.page_shift : (int)((uint32_t)t / (uint32_t)pool.page);
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
    const int64_t start = starts[b];
    const int length = seqs.length(b, pool.page);
    // at most 4096 workgroups: a step of the loop stays below 2^19 tokens
    for (int64_t at_token = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes * 4; at_token < length; at_token += (int64_t)gridDim.x * kTokens) {
        const int t = (int)at_token;
        const int p = page_of(pool, t);
        const int i0 = t - p * pool.page;
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

__device__ __forceinline__ int within(int v, int64_t most) { return v < 0 ? 0 : v < most ? v : (int)most; }

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

// What a wave has of 64 tokens, each part asked for as soon as its registers are free.  A lane's scales are those of one token, its
// quarter's number lane % 16; who needs another's takes it from that lane as an operand (a row broadcast).
template <int D, int NB>
struct Tile {
    u32x4 k[4][D / 64], v[D / 16];
    float ks[NB], vs[NB];

    // `at`: the page and head's first slot, in slots of the pool; `in`: this lane's group of sixteen in it
    __device__ __forceinline__ void load_k(const Pool &pool, int64_t at, int in, int64_t scales_at, int scales_in, int lane)
    {
        const int r = lane & 15, g = lane >> 4;
        const int8_t *const row = pool.kc + (at + in + (r & 3)) * D + g * 16;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < D / 64; ++j) k[s][j] = *reinterpret_cast<const u32x4 *>(row + 4 * s * D + 64 * j);
        const float *const scale = pool.ks + scales_at * NB + scales_in + r;
#pragma unroll
        for (int n = 0; n < NB; ++n) ks[n] = scale[(int64_t)n * pool.page];
    }
    __device__ __forceinline__ void load_v(const Pool &pool, int64_t at, int in, int lane)
    {
        const int r = lane & 15;
        const int8_t *const values = pool.vc + (at + in) * D + r * 16;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) v[t] = *reinterpret_cast<const u32x4 *>(values + t * 256);
        const float *const scale = pool.vs + at * NB + in + r;
#pragma unroll
        for (int n = 0; n < NB; ++n) vs[n] = scale[(int64_t)n * pool.page];
    }
};

// v of lane kLane of this lane's sixteen.
template <int kLane>
__device__ __forceinline__ float of_lane(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x150 + kLane, 0xf, 0xf, false));
}

template <int... kNumbers, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, kNumbers...>, F f)
{
    (f(std::integral_constant<int, kNumbers>{}), ...);
}

// A row's reference is its maximum so far or up to 2^kSlack below: it moves, and the sums with it, when a score is further above.
constexpr float kSlack = 8.0f;

// The rows of a wave: their q, statistics and sums.
template <int D, int NB, int R>
struct Rows {
    bf16x8 q[R][D / 32];
    v4f o[R][D / 16];
    float base[R], total[R];        // the reference, -inf before the first token; this lane's part of the sum
    int low[R], high[R];            // tokens seen: low < t <= high

    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int n = 0; n < R; ++n) {
            base[n] = -__builtin_inff();
            total[n] = 0.0f;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) o[n][t] = v4f{0, 0, 0, 0};
        }
    }

    // Scores of the tile's tokens, in units of log2.  Its keys are free afterwards.
    __device__ __forceinline__ void scores(const Tile<D, NB> &tile, float scale, float (&score)[R][16]) const
    {
        float ks[NB];
#pragma unroll
        for (int m = 0; m < NB; ++m) ks[m] = tile.ks[m] * scale;
        each_of(std::make_integer_sequence<int, 4>{}, [&](auto number) {
            constexpr int s = decltype(number)::value;
            v4f dot[R][NB];
#pragma unroll
            for (int n = 0; n < R; ++n)
#pragma unroll
                for (int m = 0; m < NB; ++m) dot[n][m] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                constexpr int kPer = D / 64 / NB;
                const bf16x8 a0 = widen_codes(tile.k[s][j].x, tile.k[s][j].y), a1 = widen_codes(tile.k[s][j].z, tile.k[s][j].w);
#pragma unroll
                for (int n = 0; n < R; ++n) {
                    v4f &to = dot[n][j / kPer];
                    to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, q[n][2 * j], to, 0, 0, 0);
                    to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, q[n][2 * j + 1], to, 0, 0, 0);
                }
            }
            each_of(std::make_integer_sequence<int, 4>{}, [&](auto element) {
                constexpr int i = decltype(element)::value;
#pragma unroll
                for (int n = 0; n < R; ++n) {
                    float sum = dot[n][0][i] * of_lane<4 * s + i>(ks[0]);
#pragma unroll
                    for (int m = 1; m < NB; ++m) sum = __builtin_fmaf(dot[n][m][i], of_lane<4 * s + i>(ks[m]), sum);
                    score[n][4 * s + i] = sum;
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    }

    // Takes the tile in.  `first`: the first token of this lane's sixteen; masked, the same for the wave: some row may not see
    // some token.
    __device__ __forceinline__ void add(const Tile<D, NB> &tile, float (&score)[R][16], int first, bool there, bool masked)
    {
        bf16x8 p[R][NB][2];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            int from = 0;               // seen: 0 <= token - from < count, counted from this lane's first
            uint32_t count = 16;
            if (masked) {
                const int lo = low[n] + 1 - first, hi = high[n] + 1 - first;
                from = lo < 0 ? 0 : lo < 16 ? lo : 16;
                const int to = hi < 0 ? 0 : hi < 16 ? hi : 16;
                count = there && to > from ? to - from : 0;
#pragma unroll
                for (int t = 0; t < 16; ++t) score[n][t] = (uint32_t)(t - from) < count ? score[n][t] : -__builtin_inff();
            }
            float most = __builtin_fmaxf(score[n][0], score[n][1]);
#pragma unroll
            for (int t = 2; t < 16; t += 2) most = __builtin_fmaxf(__builtin_fmaxf(score[n][t], score[n][t + 1]), most);
            most = quarters_max(most);
            if (__any(most > base[n] + kSlack)) {
                const float now = __builtin_fmaxf(base[n], most);
                const float fade = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(base[n] - now);
                base[n] = now;
                total[n] *= fade;
#pragma unroll
                for (int t = 0; t < D / 16; ++t) o[n][t] *= fade;
            }
            const float reference = base[n] == -__builtin_inff() ? 0.0f : base[n];
            float sums[2] = {0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                score[n][t] = __builtin_amdgcn_exp2f(score[n][t] - reference);
                sums[t % 2] += score[n][t];
            }
            total[n] += sums[0] + sums[1];
            each_of(std::make_integer_sequence<int, NB>{}, [&](auto number) {
                constexpr int m = decltype(number)::value;
                float e[16];
                each_of(std::make_integer_sequence<int, 16>{}, [&](auto token) {
                    constexpr int t = decltype(token)::value;
                    e[t] = score[n][t] * of_lane<t>(tile.vs[m]);
                });
                if (masked) {           // what is not seen may have any scale
                    asm volatile("" : "+v"(from), "+v"(count));     // the comparisons again: kept, they would be 32 scalar registers
#pragma unroll
                    for (int t = 0; t < 16; ++t) e[t] = (uint32_t)(t - from) < count ? e[t] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 w = {narrow_bf16x2(e[8 * j], e[8 * j + 1]), narrow_bf16x2(e[8 * j + 2], e[8 * j + 3]),
                                     narrow_bf16x2(e[8 * j + 4], e[8 * j + 5]), narrow_bf16x2(e[8 * j + 6], e[8 * j + 7])};
                    p[n][m][j] = __builtin_bit_cast(bf16x8, w);
                }
            });
        }
        // codes are widened as they are used: early, they would be twice the registers
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
            constexpr int kPer = D / 16 / NB;
            if (t % 2 == 0) __builtin_amdgcn_sched_barrier(0);
            const bf16x8 a0 = widen_codes(tile.v[t].x, tile.v[t].y), a1 = widen_codes(tile.v[t].z, tile.v[t].w);
#pragma unroll
            for (int n = 0; n < R; ++n) {
                o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, p[n][t / kPer][0], o[n][t], 0, 0, 0);
                o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, p[n][t / kPer][1], o[n][t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
};

// Where a lane's keys and values of a tile are: its page and head's first slot, and its group of sixteen there.
struct Place {
    int64_t k_at, v_at;
    int k_in, v_in;
    bool there;
};

// Waves of a workgroup: on the same rows and different tokens (kTokens), their results joined at the end, or on
// different rows.
template <int D, int NB, int R, bool kTokens>
__global__ __launch_bounds__(256, R == 1 && D <= 128 ? 2 : 1) void attention_kernel(const AttentionCall call, const Sequences seqs,
                                                                                    const Pool pool)
{
    constexpr int W = 4;
    constexpr float kNone = -__builtin_inff();
    constexpr int kPitch = D + 4;           // of a row of results in LDS, whose statistics are behind it
    __shared__ float joined[kTokens ? W / 2 : 1][kTokens ? R * 16 : 1][kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int b = blockIdx.z, split = blockIdx.y / (uint32_t)pool.heads, h = blockIdx.y - split * pool.heads;
    const int q0 = within(call.q_starts[b], call.q_rows), queries = within(call.q_starts[b + 1], call.q_rows) - q0;
    const int length = seqs.length(b, pool.page);
    // this split's tokens: whole tiles; a sequence longer than the host knew has longer splits
    int chunk = call.chunk;
    if ((int64_t)chunk * call.splits < length) chunk = (int)((uint32_t)(length + call.splits - 1) / (uint32_t)call.splits + 63 & ~63u);
    const int64_t split_from = (int64_t)split * chunk;
    const int split_first = split_from < length ? (int)split_from : length;
    const int split_last = split_from + chunk < length ? (int)split_from + chunk : length;

    const int32_t *const table = seqs.table + b * seqs.width;
    // page numbers of a tile from t0 on, of this lane's keys and values; -1 past the table
    auto pages_of = [&](int t0, int &k_id, int &v_id) {
        const int k_p = page_of(pool, t0 + 16 * (r >> 2)), v_p = page_of(pool, t0 + 16 * g);
        k_id = k_p < seqs.width ? table[k_p] : -1;
        v_id = v_p < seqs.width ? table[v_p] : -1;
    };
    auto place_of = [&](int t0, int k_id, int v_id) {
        Place p;
        const int k_t = t0 + 16 * (r >> 2), v_t = t0 + 16 * g;
        p.there = v_id >= 0 && v_id < pool.pages;
        if (k_id < 0 || k_id >= pool.pages) k_id = 0;       // loaded, not seen
        if (!p.there) v_id = 0;
        p.k_at = pool.place(k_id, h) * pool.page;
        p.v_at = pool.place(v_id, h) * pool.page;
        p.k_in = k_t - page_of(pool, k_t) * pool.page;
        p.v_in = v_t - page_of(pool, v_t) * pool.page;
        return p;
    };

    const int rows = queries * call.group;
    constexpr int kRows = (kTokens ? 1 : W) * R * 16;
    const int row_tiles = (rows + kRows - 1) / kRows;
    for (int turn = blockIdx.x; turn < row_tiles; turn += gridDim.x) {
        // with causal rows the last ones are the longest: they begin first
        const int tile_row = (kTokens ? turn : row_tiles - 1 - turn) * kRows;
        const int row0 = tile_row + (kTokens ? 0 : wave * R * 16);
        auto query_of = [&](int row) { return (int)((uint32_t)(row < rows ? row : rows - 1) / (uint32_t)call.group); };
        Rows<D, NB, R> mine;
        mine.start();
        int64_t place_out[R];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            const int row = row0 + n * 16 + r < rows ? row0 + n * 16 + r : rows - 1;
            const int i = query_of(row), member = h * call.group + (row - i * call.group);
            const int at = length - queries + i;
            mine.high[n] = call.causal ? (at < -1 ? -1 : at) : length - 1;
            mine.low[n] = call.window && at >= call.window ? at - call.window : -1;
            place_out[n] = (int64_t)(q0 + i) * call.q_heads + member;
            const uint16_t *const from = call.q + (q0 + i) * call.q_row + member * call.q_head + g * 16;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                mine.q[n][j] = *reinterpret_cast<const bf16x8 *>(from + (j / 2) * 64 + (j % 2) * 8);
        }
        // what any row of the wave sees of this split, and what all of them see
        int first = split_first, last = split_last;
        int all_from = 0, all_to = length;
        if (call.causal) {
            const int at_first = length - queries + query_of(row0), at_last = length - queries + query_of(row0 + R * 16 - 1);
            if (at_last + 1 < last) last = at_last + 1;
            all_to = at_first + 1;
            if (call.window && at_last >= call.window) {
                if (at_first >= call.window && at_first - call.window + 1 > first) first = (at_first - call.window + 1) & ~63;
                all_from = at_last - call.window + 1;
            }
        }
        constexpr int kStep = (kTokens ? W : 1) * 64;
        int t0 = first + (kTokens ? wave * 64 : 0);
        if (t0 < last) {
            Tile<D, NB> tile;
            int k_id, v_id;
            pages_of(t0, k_id, v_id);
            Place place = place_of(t0, k_id, v_id);
            tile.load_k(pool, place.k_at, place.k_in, place.v_at, place.v_in, lane);
            tile.load_v(pool, place.v_at, place.v_in, lane);
            bool there = place.there;
            pages_of(t0 + kStep, k_id, v_id);
            do {
                // past the end the next tile is one of another split, or of no page: loaded, not used
                const Place next = place_of(t0 + kStep, k_id, v_id);
                float score[R][16];
                mine.scores(tile, call.scale, score);
                tile.load_k(pool, next.k_at, next.k_in, next.v_at, next.v_in, lane);
                pages_of(t0 + 2 * kStep, k_id, v_id);
                __builtin_amdgcn_sched_barrier(0);
                mine.add(tile, score, t0 + 16 * g, there, !(t0 >= all_from && t0 + 64 <= all_to && __all(there)));
                tile.load_v(pool, next.v_at, next.v_in, lane);
                there = next.there;
                t0 += kStep;
            } while (t0 < last);
        }
#pragma unroll
        for (int n = 0; n < R; ++n) mine.total[n] = quarters_sum(mine.total[n]);

        if constexpr (kTokens) {            // join the four waves: two halves, then one
            auto give = [&](int to) {
#pragma unroll
                for (int n = 0; n < R; ++n) {
#pragma unroll
                    for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(&joined[to][n * 16 + r][t * 16 + 4 * g]) = mine.o[n][t];
                    if (g == 0) {
                        joined[to][n * 16 + r][D] = mine.base[n];
                        joined[to][n * 16 + r][D + 1] = mine.total[n];
                    }
                }
            };
            auto take = [&](int from) {
#pragma unroll
                for (int n = 0; n < R; ++n) {
                    const float base = joined[from][n * 16 + r][D], total = joined[from][n * 16 + r][D + 1];
                    const float now = __builtin_fmaxf(mine.base[n], base), reference = now == kNone ? 0.0f : now;
                    const float fade = __builtin_amdgcn_exp2f(mine.base[n] - reference), other = __builtin_amdgcn_exp2f(base - reference);
                    mine.base[n] = now;
                    mine.total[n] = mine.total[n] * fade + total * other;
#pragma unroll
                    for (int t = 0; t < D / 16; ++t)
                        mine.o[n][t] = mine.o[n][t] * fade + *reinterpret_cast<const v4f *>(&joined[from][n * 16 + r][t * 16 + 4 * g]) * other;
                }
            };
            __syncthreads();                // the last rows' results have been read
            if (wave >= 2) give(wave - 2);
            __syncthreads();
            if (wave < 2) take(wave);
            __syncthreads();
            if (wave == 1) give(0);
            __syncthreads();
            if (wave == 0) take(0);
        }
        if (kTokens && wave != 0) continue;
#pragma unroll
        for (int n = 0; n < R; ++n) {
            if (row0 + n * 16 + r >= rows) continue;
            if (call.splits > 1) {
                const int64_t at = split * call.q_rows * call.q_heads + place_out[n];
#pragma unroll
                for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(call.part + at * D + t * 16 + 4 * g) = mine.o[n][t];
                if (g == 0) {
                    float *const stats = call.part + call.splits * call.q_rows * call.q_heads * D + at * 2;
                    stats[0] = mine.base[n];
                    stats[1] = mine.total[n];
                }
            } else {
                const float inverse = ends_with(mine.total[n]);
#pragma unroll
                for (int t = 0; t < D / 16; ++t) {
                    const v4f o = mine.o[n][t] * inverse;
                    *reinterpret_cast<u32x2 *>(call.out + place_out[n] * D + t * 16 + 4 * g) = u32x2{narrow_bf16x2(o[0], o[1]), narrow_bf16x2(o[2], o[3])};
                }
                if (call.lse && g == 0) call.lse[place_out[n]] = log_sum(mine.base[n], mine.total[n]);
            }
        }
    }
}

// Joins the splits of an output row, a workgroup each: D / 4 lanes take a split, the others other splits, and the parts are
// added in order.  Little is read and much waited for: what can be asked for at once is (the splits' statistics one after
// the other: 17.5 us for 64 splits).
constexpr int kMostSplits = 64;         // a lane each

template <int D>
__global__ __launch_bounds__(256) void join_kernel(const AttentionCall call, int32_t sequences)
{
    constexpr int kLanes = D / 4, kParts = 256 / kLanes, kRounds = kMostSplits / kParts;
    constexpr float kNone = -__builtin_inff();
    __shared__ v4f part[kParts][kLanes];
    const int64_t all = call.q_rows * call.q_heads, at = blockIdx.x;
    const int row = (int)(blockIdx.x / (uint32_t)call.q_heads);
    const int from = call.q_starts[0], to = call.q_starts[sequences];
    const int mine = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, split = threadIdx.x & 63;
    const float2 stat = split < call.splits ? reinterpret_cast<const float2 *>(call.part + call.splits * all * D)[split * all + at]
                                            : float2{kNone, 0.0f};
    const float *const sums = call.part + at * D + lane * 4;
    v4f o[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int s = mine + i * kParts;
        o[i] = s < call.splits ? *reinterpret_cast<const v4f *>(sums + s * all * D) : v4f{0, 0, 0, 0};
    }
    loads_first();
    if (row < from || row >= to) return;        // a row of no sequence
    float now = stat.x;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) now = __builtin_fmaxf(now, __shfl_xor(now, step));
    const float weight = __builtin_amdgcn_exp2f(stat.x - (now == kNone ? 0.0f : now));
    float total = stat.y * weight;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) total += __shfl_xor(total, step);
    v4f acc = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kRounds; ++i) acc += o[i] * __shfl(weight, mine + i * kParts);
    part[mine][lane] = acc;
    __syncthreads();
    if (mine != 0) return;
#pragma unroll
    for (int p = 1; p < kParts; ++p) acc += part[p][lane];
    acc *= ends_with(total);
    *reinterpret_cast<u32x2 *>(call.out + at * D + lane * 4) = u32x2{narrow_bf16x2(acc[0], acc[1]), narrow_bf16x2(acc[2], acc[3])};
    if (call.lse && lane == 0) call.lse[at] = log_sum(now, total);
}

}  // namespace cache
}  // namespace equarx
