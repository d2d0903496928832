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
// A lane has eight elements of T = 4 consecutive tokens of the call, or of one; dim / 8 lanes a head.  Keys are written eight
// bytes at a time.  An element's value codes of sixteen slots are sixteen bytes: where a wave's tokens are whole such groups
// its quarters, four tokens each, exchange words and write them whole; else four tokens are written together where they lie
// in one group from a multiple of four on, and byte by byte where they do not.  Memory is the bound: 16384 tokens of 8 heads of 128
// in 19.8 us (5.2 TB/s), 23.0 without the exchange.

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

// Word i of quarter q of a wave to word q of quarter i.
__device__ __forceinline__ u32x4 exchange_quarters(const u32x4 &w)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w.x, w.z, false, false), b = __builtin_amdgcn_permlane32_swap(w.y, w.w, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

template <int D, int B, int T>
__global__ __launch_bounds__(256) void write_kernel(Global<const uint16_t> k, Global<const uint16_t> v,
                                                    Global<const int64_t> slots, int64_t k_row, int64_t v_row,
                                                    int32_t tokens, int64_t k_head, int64_t v_head, const Pool pool)
{
    constexpr int kLanes = D / 8, kBlocks = D / B, G = B / 8;
    const int h = blockIdx.y;
    int part = threadIdx.x / kLanes;
    if (T == 4 && D == 64) part = (part & ~7) + (part >> 1 & 3) + (part & 1) * 4;       // a quarter's tokens: of two groups
    const int t0 = (blockIdx.x * (256 / kLanes) + part) * T;
    const int d = threadIdx.x % kLanes * 8;
    const int64_t space = pool.pages * pool.page;
    u32x4 kx[T], vx[T];
    int64_t slot[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int t = t0 + i < tokens ? t0 + i : tokens - 1;
        slot[i] = t0 + i < tokens ? slots[t] : -1;
        if (slot[i] >= space) slot[i] = -1;
        kx[i] = *reinterpret_cast<const u32x4 *>(k + t * k_row + h * k_head + d);
        vx[i] = *reinterpret_cast<const u32x4 *>(v + t * v_row + h * v_head + d);
    }
    loads_first();
    u32x2 vw[T];
    int64_t at[T];
    int in_page[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
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
    if constexpr (T == 4) {
        const bool together = slot[0] >= 0 && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 &&
                              slot[3] == slot[0] + 3;
        int8_t *const group = pool.vc + at[0] * pool.page * D + (int64_t)(in_page[0] & ~15) * D;
        u32x4 w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = transpose4(vw[0][j], vw[1][j], vw[2][j], vw[3][j]);
        if constexpr (D <= 128) {
            // this lane's tokens follow those of the quarters before it, from a group's first on
            const int quarter = threadIdx.x >> 4 & 3;
            const int64_t first = __shfl(slot[0], threadIdx.x & 15);
            if (__all(together && (first & 15) == 0 && slot[0] == first + 4 * quarter)) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<u32x4 *>(group + (d + 4 * j + quarter) * 16) = exchange_quarters(w[j]);
                return;
            }
        }
        if (together) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<uint32_t *>(group + d * 16 + (in_page[0] & 15) + (4 * j + i) * 16) = w[j][i];
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < T; ++i) {
        if (slot[i] < 0) continue;
        int8_t *const to = pool.vc + at[i] * pool.page * D + (int64_t)(in_page[i] & ~15) * D + d * 16 + (in_page[i] & 15);
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j * 16] = (int8_t)(vw[i][j / 4] >> (8 * (j % 4)));
    }
}

// ---------------------------------------------------------------- reading back
// A lane has eight elements of four tokens from a multiple of four on, dim / 8 lanes a head.  Memory is the bound: the tokens
// above back in 19.0 us (5.4 TB/s).

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
// A code is exact in bf16; scales join in fp32, the keys' on the scores, the values' on the probabilities.  These products
// go to the matrix instructions as sums of two bf16: rounded to one, 2^-9 of each, their error is as large as that of the result's
// own rounding, and f16 has not the range for the small ones.  Running maximum and sum per row; the sum stays split over the
// quarters until the end.

struct AttentionCall {
    const uint16_t *q;
    int64_t q_row, q_head;
    const int32_t *q_starts;
    uint16_t *out;
    float *lse;
    float *part;                // parts of rows to be joined, sums and then statistics
    int64_t q_rows;
    int32_t q_heads, group;
    float scale;                // times log2(e)
    int32_t causal, window;
    int32_t chunk, splits;      // waves on rows: a split's tokens, a multiple of 64
    int32_t sequences;
    int32_t tiles_last;         // waves on rows: the grid's third dimension is tiles of rows, not sequences
};

__device__ __forceinline__ int within(int v, int64_t most) { return v < 0 ? 0 : v < most ? v : (int)most; }

// A row's maximum is -inf until it sees a token, and kLeast at least from then on: so a row that saw nothing is told from one all of
// whose scores are -inf.  The first is zeros; the second's sums stay 0, and its result is 0 / 0.
constexpr float kLeast = -3.402823466e38f;

// The factor that ends a row, and its log sum of exponentials.
__device__ __forceinline__ float ends_with(float top, float total) { return top == -__builtin_inff() ? 0.0f : 1.0f / total; }
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

// Eight numbers as the sums of two bf16, the first their upper halves: to 2^-16 of each.
__device__ __forceinline__ void split_in_two(const float *e, bf16x8 &upper, bf16x8 &rest)
{
    u32x4 u, r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(e[2 * i]), b = __float_as_uint(e[2 * i + 1]);
        u[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        r[i] = narrow_bf16x2(e[2 * i] - __uint_as_float(a & 0xffff0000u), e[2 * i + 1] - __uint_as_float(b & 0xffff0000u));
    }
    upper = __builtin_bit_cast(bf16x8, u);
    rest = __builtin_bit_cast(bf16x8, r);
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

// A block with this is jumped over where it is not due; else the compiler makes selects of it, for every tile.
__device__ __forceinline__ void stay_a_branch() { asm volatile(""); }

// v of lane kLane of this lane's sixteen: a part of the product that takes it.
template <int kLane>
__device__ __forceinline__ float of_lane(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x150 + kLane, 0xf, 0xf, true));
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
                    for (int m = 1; m < NB; ++m) sum += dot[n][m][i] * of_lane<4 * s + i>(ks[m]);
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
        bf16x8 p[R][NB][2], rest[R][NB][2];
#pragma unroll
        for (int n = 0; n < R; ++n) {
            int from = 0;               // seen: 0 <= token - from < count, counted from this lane's first
            uint32_t count = 16;
            float least = kLeast;
            if (masked) {
                stay_a_branch();
                const int lo = low[n] + 1 - first, hi = high[n] + 1 - first;
                from = lo < 0 ? 0 : lo < 16 ? lo : 16;
                const int to = hi < 0 ? 0 : hi < 16 ? hi : 16;
                count = there && to > from ? to - from : 0;
                least = count ? kLeast : -__builtin_inff();
#pragma unroll
                for (int t = 0; t < 16; ++t) score[n][t] = (uint32_t)(t - from) < count ? score[n][t] : -__builtin_inff();
            }
            float most = least;
#pragma unroll
            for (int t = 0; t < 16; t += 2) most = __builtin_fmaxf(__builtin_fmaxf(score[n][t], score[n][t + 1]), most);
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
                for (int j = 0; j < 2; ++j) split_in_two(e + 8 * j, p[n][m][j], rest[n][m][j]);
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
                o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, rest[n][t / kPer][0], o[n][t], 0, 0, 0);
                o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, rest[n][t / kPer][1], o[n][t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
};

// Rows `first` .. first + R * 16 - 1 of a sequence and key head: row n * 16 + lane % 16 as a query and its head, past the end the last.
struct Row {
    int query, head;
    __device__ __forceinline__ Row(const AttentionCall &call, int queries, int h, int row)
    {
        const int rows = queries * call.group;
        if (row >= rows) row = rows - 1;
        query = (int)((uint32_t)row / (uint32_t)call.group);
        head = h * call.group + (row - query * call.group);
    }
};

template <int D, int NB, int R>
__device__ __forceinline__ void load_q(Rows<D, NB, R> &mine, const AttentionCall &call, int q0, int queries, int h, int first, int lane)
{
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const Row row(call, queries, h, first + n * 16 + (lane & 15));
        const uint16_t *const from = call.q + (q0 + row.query) * call.q_row + row.head * call.q_head + (lane >> 4) * 16;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) mine.q[n][j] = *reinterpret_cast<const bf16x8 *>(from + (j / 2) * 64 + (j % 2) * 8);
    }
}

// What the rows see, nothing summed yet; and where their results go.
template <int D, int NB, int R>
__device__ __forceinline__ void start_rows(Rows<D, NB, R> &mine, const AttentionCall &call, int queries, int length, int h, int first,
                                           int lane)
{
    mine.start();
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const int at = length - queries + Row(call, queries, h, first + n * 16 + (lane & 15)).query;
        mine.high[n] = call.causal ? (at < -1 ? -1 : at) : length - 1;
        mine.low[n] = call.window && at >= call.window ? at - call.window : -1;
    }
}

__device__ __forceinline__ int64_t place_of_row(const AttentionCall &call, int q0, const Row &row)
{
    return (int64_t)(q0 + row.query) * call.q_heads + row.head;
}

// The tokens that any of some consecutive rows sees, first .. last - 1 with first a multiple of 64, and those that all see.
struct Span {
    int first, last, all_from, all_to;
};

__device__ __forceinline__ Span span_of(const AttentionCall &call, int queries, int length, int row_first, int row_last)
{
    const int rows = queries * call.group;
    Span s{0, length, 0, length};
    if (call.causal) {
        if (row_last >= rows) row_last = rows - 1;
        if (row_first >= rows) row_first = rows - 1;
        const int at_first = length - queries + (int)((uint32_t)row_first / (uint32_t)call.group);
        const int at_last = length - queries + (int)((uint32_t)row_last / (uint32_t)call.group);
        s.last = at_last + 1 < 0 ? 0 : at_last + 1;
        s.all_to = at_first + 1;
        if (call.window) {
            if (at_first >= call.window) s.first = (at_first - call.window + 1) & ~63;
            if (at_last >= call.window) s.all_from = at_last - call.window + 1;
        }
    }
    return s;
}

// Where a lane's keys and values of the tile from token t on are: page numbers, -1 past the table; a page and head's first slot;
// a group there.
struct PageIds {
    int k, v;
    __device__ __forceinline__ PageIds(const Pool &pool, const int32_t *table, int64_t width, int t, int lane)
    {
        const int k_p = page_of(pool, t + 16 * ((lane & 15) >> 2)), v_p = page_of(pool, t + 16 * (lane >> 4));
        k = k_p < width ? table[k_p] : -1;
        v = v_p < width ? table[v_p] : -1;
    }
};

struct Place {
    int64_t k_at, v_at;
    int k_in, v_in;
    bool there;
    __device__ __forceinline__ Place(const Pool &pool, PageIds ids, int h, int t, int lane)
    {
        const int k_t = t + 16 * ((lane & 15) >> 2), v_t = t + 16 * (lane >> 4);
        there = ids.v >= 0 && ids.v < pool.pages;
        if (ids.k < 0 || ids.k >= pool.pages) ids.k = 0;        // loaded, not seen
        if (!there) ids.v = 0;
        k_at = pool.place(ids.k, h) * pool.page;
        v_at = pool.place(ids.v, h) * pool.page;
        k_in = k_t - page_of(pool, k_t) * pool.page;
        v_in = v_t - page_of(pool, v_t) * pool.page;
    }
};

// Takes the tiles t0, t0 + kStep, ... below `last` in.
template <int kStep, int D, int NB, int R>
__device__ __forceinline__ void walk(Rows<D, NB, R> &mine, const Pool &pool, const int32_t *table, int64_t width, int h, float scale,
                                     int t0, int last, const Span &span, int lane)
{
    if (t0 >= last) return;
    Tile<D, NB> tile;
    const Place place(pool, PageIds(pool, table, width, t0, lane), h, t0, lane);
    tile.load_k(pool, place.k_at, place.k_in, place.v_at, place.v_in, lane);
    tile.load_v(pool, place.v_at, place.v_in, lane);
    bool there = place.there;
    PageIds ids(pool, table, width, t0 + kStep, lane);
    do {
        // past the end the next tile is one of another part, or of no page: loaded, not used
        const Place next(pool, ids, h, t0 + kStep, lane);
        float score[R][16];
        mine.scores(tile, scale, score);
        tile.load_k(pool, next.k_at, next.k_in, next.v_at, next.v_in, lane);
        ids = PageIds(pool, table, width, t0 + 2 * kStep, lane);
        __builtin_amdgcn_sched_barrier(0);
        mine.add(tile, score, t0 + 16 * (lane >> 4), there, !(t0 >= span.all_from && t0 + 64 <= span.all_to && __all(there)));
        tile.load_v(pool, next.v_at, next.v_in, lane);
        there = next.there;
        t0 += kStep;
    } while (t0 < last);
}

// Row n's results, to the output or to a part: sums at `part`, statistics at `stats`.
template <int D, int NB, int R>
__device__ __forceinline__ void end_row(const Rows<D, NB, R> &mine, int n, const AttentionCall &call, int64_t place_out, int lane)
{
    const int g = lane >> 4;
    const float inverse = ends_with(mine.base[n], mine.total[n]);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
        const v4f o = mine.o[n][t] * inverse;
        *reinterpret_cast<u32x2 *>(call.out + place_out * D + t * 16 + 4 * g) = u32x2{narrow_bf16x2(o[0], o[1]), narrow_bf16x2(o[2], o[3])};
    }
    if (call.lse && g == 0) call.lse[place_out] = log_sum(mine.base[n], mine.total[n]);
}

template <int D, int NB, int R>
__device__ __forceinline__ void part_row(const Rows<D, NB, R> &mine, int n, float *part, float2 *stats, int lane)
{
    const int g = lane >> 4;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(part + t * 16 + 4 * g) = mine.o[n][t];
    if (g == 0) *stats = float2{mine.base[n], mine.total[n]};
}

// ---- many rows: the waves of a workgroup have 32 different ones each
// Here the matrix unit and what comes between its instructions are the bound, so codes are widened once for a workgroup: wave w takes
// the keys and values of sixteen tokens of 64, as bf16 they wait in LDS (two buffers: the next tile's are written, and the one
// after that asked for, while this one's are used) in the order in which the lanes of a 32x32x16 instruction read them.
// (2 x 2048 rows of 32 heads at the end of 8192 tokens, blocks of 64: every wave widening all for itself, 16x16x32, 1055 us;
// this 629, 0.60 PFLOP/s, of which 130 are for probabilities as two bf16.  Two thirds of the cycles issue vector instructions -- 620
// a wave and tile, the exponentials four times as long as others --, a third have a matrix instruction under way, and few both.  Of
// the LDS cycles a third are conflicts: the four lanes of a token store quarters of its keys that lie in the same banks.)
//
// As above with 32 for 16: the tokens of an instruction's rows are chosen so that S^T leaves lane (row c = l % 32, half h = l / 32)
// with 16 consecutive tokens 16 h .. of the 32, row 8 j + 4 h + i being token 16 h + 4 j + i, and O^T += V^T P^T takes eight of
// these as they are.
// Grid: heads x splits, then sequences and tiles of rows in either order: tiles of one head, which read the same tokens, are on one
// XCD as a rule.  Parts: [splits][q_rows][q_heads].

typedef float v16f __attribute__((ext_vector_type(16)));

template <int D, int NB>
struct RowsTile {
    // A tile in LDS: the keys of bf16, the values, then scales [keys, values][block][token] and whether each sixteen tokens have
    // a page.
    static constexpr int kKeys = D * 128, kScales = 2 * kKeys, kThere = kScales + 2 * NB * 256, kBytes = kThere + 16;
    static constexpr int kPieces = D / 64;                          // of 16 codes, a lane's keys and its values
    static constexpr int kLoads = NB < 4 ? 1 : 2;                   // of scales, a lane's: 16 tokens' are 32 NB

    // What a wave's lane has of the wave's sixteen tokens on the way: lane l 1/4 of the keys of token l / 4, and the sixteen
    // values of elements l, l + 64, ...; and scales of token l % 16.  They are in one page, found a tile ahead.
    u32x4 k[kPieces], v[kPieces];
    float scale[kLoads];
    bool there;
    int id;

    static __device__ __forceinline__ bool of_values(int i, int lane) { return NB == 1 ? lane >> 4 & 1 : NB == 2 ? lane >> 5 : i; }
    static __device__ __forceinline__ int block_of(int lane) { return (lane >> 4) & (NB - 1); }

    __device__ __forceinline__ void find(const Pool &pool, const int32_t *table, int64_t width, int t)
    {
        const int p = page_of(pool, t);
        id = p < width ? table[p] : -1;
    }

    __device__ __forceinline__ void load(const Pool &pool, int h, int t, int lane)
    {
        const int page = __builtin_amdgcn_readfirstlane(id), in = t - page_of(pool, t) * pool.page;
        there = page >= 0 && page < pool.pages;
        const int64_t first = pool.place(there ? page : 0, h) * pool.page, at = first + in;      // no page: any one's, not seen
        const int8_t *const keys = pool.kc + at * D + (lane >> 2) * D + (lane & 3) * (D / 4);
        const int8_t *const values = pool.vc + at * D + lane * 16;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            k[i] = *reinterpret_cast<const u32x4 *>(keys + 16 * i);
            v[i] = *reinterpret_cast<const u32x4 *>(values + 1024 * i);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            scale[i] = (of_values(i, lane) ? pool.vs : pool.ks)[first * NB + in + block_of(lane) * pool.page + (lane & 15)];
    }

    // The codes, widened, into a buffer; the keys' scales with the call's.  Keys: fragment (32 tokens, 16 elements) is 1 KB, lane
    // after lane.  Values: fragment (32 elements, 32 tokens, 16 of them) the same.
    __device__ __forceinline__ void store(uint8_t *buffer, float key_scale, int wave, int lane) const
    {
        const int token = lane >> 2, quarter = lane & 3, place = 8 * (token >> 2) + 4 * (wave & 1) + (token & 3);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            uint8_t *const keys = buffer + (wave >> 1) * (D * 64) + (quarter * kPieces + i) * 1024 + place * 16;
            *reinterpret_cast<bf16x8 *>(keys) = widen_codes(k[i].x, k[i].y);
            *reinterpret_cast<bf16x8 *>(keys + 512) = widen_codes(k[i].z, k[i].w);
            uint8_t *const values = buffer + kKeys + ((2 * i + (lane >> 5)) * 4 + (wave >> 1) * 2) * 1024 + ((wave & 1) * 32 + (lane & 31)) * 16;
            *reinterpret_cast<bf16x8 *>(values) = widen_codes(v[i].x, v[i].y);
            *reinterpret_cast<bf16x8 *>(values + 1024) = widen_codes(v[i].z, v[i].w);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool values = of_values(i, lane);
            reinterpret_cast<float *>(buffer + kScales)[(values * NB + block_of(lane)) * 64 + 16 * wave + (lane & 15)] =
                values ? scale[i] : scale[i] * key_scale;
        }
        if (lane == 0) reinterpret_cast<int32_t *>(buffer + kThere)[wave] = there;
    }
};

__device__ __forceinline__ float halves_max(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D, int NB>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void attention_rows_kernel(const AttentionCall call, const Sequences seqs,
                                                                               const Pool pool)
{
    constexpr int kRows = 128;
    __shared__ __align__(16) uint8_t lds[2][RowsTile<D, NB>::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, half = lane >> 5;
    const int b = call.tiles_last ? blockIdx.y : blockIdx.z, split = blockIdx.x / (uint32_t)pool.heads, h = blockIdx.x - split * pool.heads;
    const int first_turn = call.tiles_last ? blockIdx.z : blockIdx.y, turns = call.tiles_last ? gridDim.z : gridDim.y;
    const int q0 = within(call.q_starts[b], call.q_rows), queries = within(call.q_starts[b + 1], call.q_rows) - q0;
    const int length = seqs.length(b, pool.page);
    const int32_t *const table = seqs.table + b * seqs.width;
    // this split's tokens: whole tiles; a sequence longer than the host knew has longer splits
    int chunk = call.chunk;
    if ((int64_t)chunk * call.splits < length) chunk = (int)((uint32_t)(length + call.splits - 1) / (uint32_t)call.splits + 63 & ~63u);
    const int64_t split_from = (int64_t)split * chunk;

    const int rows = queries * call.group, row_tiles = (rows + kRows - 1) / kRows;
    for (int turn = first_turn; turn < row_tiles; turn += turns) {
        const int tile_row = (row_tiles - 1 - turn) * kRows;        // with causal rows the last ones are the longest: first
        const int row0 = tile_row + wave * 32;
        const Row row(call, queries, h, row0 + r);
        bf16x8 q[D / 16];
        {
            const uint16_t *const from = call.q + (q0 + row.query) * call.q_row + row.head * call.q_head + half * 8;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) q[j] = *reinterpret_cast<const bf16x8 *>(from + 16 * j);
        }
        const int at = length - queries + row.query;
        const int high = call.causal ? (at < -1 ? -1 : at) : length - 1;        // seen: low < token <= high
        const int low = call.window && at >= call.window ? at - call.window : -1;
        // what any row of the workgroup sees of this split, and what all of the wave's see
        Span span = span_of(call, queries, length, tile_row, tile_row + kRows - 1);
        const Span mine = span_of(call, queries, length, row0, row0 + 31);
        if (split_from > span.first) span.first = split_from < length ? (int)split_from : length;
        if (split_from + chunk < span.last) span.last = (int)split_from + chunk;

        v16f o[D / 32];
#pragma unroll
        for (int t = 0; t < D / 32; ++t) o[t] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        float base = -__builtin_inff(), total = 0.0f;
        RowsTile<D, NB> next;
        int cur = 0;
        if (span.first < span.last) {
            __syncthreads();                    // the last rows' tiles have been read
            next.find(pool, table, seqs.width, span.first + 16 * wave);
            next.load(pool, h, span.first + 16 * wave, lane);
            next.store(lds[0], call.scale, wave, lane);
            next.find(pool, table, seqs.width, span.first + 16 * wave + 64);
        }
        for (int t0 = span.first; t0 < span.last; t0 += 64) {
            __syncthreads();                    // this tile is there for all, and the other buffer read by all
            // past the end the next tile is one of another part, or of no page: loaded, not used
            next.load(pool, h, t0 + 64 + 16 * wave, lane);
            next.find(pool, table, seqs.width, t0 + 128 + 16 * wave);
            const uint8_t *const tile = lds[cur];
            float ks[2][NB], vs[2][NB];
            bool there[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float *const scales = reinterpret_cast<const float *>(tile + RowsTile<D, NB>::kScales) + 32 * i + 16 * half + (lane & 15);
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    ks[i][m] = scales[m * 64];
                    vs[i][m] = scales[(NB + m) * 64];
                }
                there[i] = reinterpret_cast<const int32_t *>(tile + RowsTile<D, NB>::kThere)[2 * i + half];
            }
            if (row0 < rows && t0 < mine.last && t0 + 64 > mine.first) {
                const bool masked = !(t0 >= mine.all_from && t0 + 64 <= mine.all_to && __all(there[0] && there[1]));
                float score[2][16];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    v16f dot[NB];
#pragma unroll
                    for (int m = 0; m < NB; ++m) dot[m] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                    for (int n = 0; n < D / 16; ++n) {
                        constexpr int kPer = D / 16 / NB;
                        const int m = n % NB, j = m * kPer + n / NB;
                        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(tile + i * (D * 64) + j * 1024 + lane * 16);
                        dot[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[j], dot[m], 0, 0, 0);
                    }
                    each_of(std::make_integer_sequence<int, 16>{}, [&](auto token) {
                        constexpr int t = decltype(token)::value;
                        float sum = dot[0][t] * of_lane<t>(ks[i][0]);
#pragma unroll
                        for (int m = 1; m < NB; ++m) sum += dot[m][t] * of_lane<t>(ks[i][m]);
                        score[i][t] = sum;
                    });
                }
                int from[2] = {0, 0};               // seen: 0 <= token - from < count, counted from this lane's first of a block
                uint32_t count[2] = {16, 16};
                float most = kLeast;
                if (masked) {
                    stay_a_branch();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int first = t0 + 32 * i + 16 * half, lo = low + 1 - first, hi = high + 1 - first;
                        from[i] = lo < 0 ? 0 : lo < 16 ? lo : 16;
                        const int to = hi < 0 ? 0 : hi < 16 ? hi : 16;
                        count[i] = there[i] && to > from[i] ? to - from[i] : 0;
#pragma unroll
                        for (int t = 0; t < 16; ++t) score[i][t] = (uint32_t)(t - from[i]) < count[i] ? score[i][t] : -__builtin_inff();
                    }
                    most = (count[0] | count[1]) != 0 ? kLeast : -__builtin_inff();
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < 16; ++t) most = __builtin_fmaxf(most, score[i][t]);
                most = halves_max(most);
                if (__any(most > base + kSlack)) {
                    const float now = __builtin_fmaxf(base, most);
                    const float fade = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(base - now);
                    base = now;
                    total *= fade;
#pragma unroll
                    for (int t = 0; t < D / 32; ++t) o[t] *= fade;
                }
                const float reference = base == -__builtin_inff() ? 0.0f : base;
                float sums[2] = {0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        score[i][t] = __builtin_amdgcn_exp2f(score[i][t] - reference);
                        sums[t % 2] += score[i][t];
                    }
                total += sums[0] + sums[1];
                // block by block of the values' elements: one block's products are registers enough
                each_of(std::make_integer_sequence<int, NB>{}, [&](auto number) {
                    constexpr int m = decltype(number)::value, kPer = D / 32 / NB;
                    bf16x8 p[4], rest[4];
                    each_of(std::make_integer_sequence<int, 2>{}, [&](auto block) {
                        constexpr int i = decltype(block)::value;
                        float e[16];
                        each_of(std::make_integer_sequence<int, 16>{}, [&](auto token) {
                            constexpr int t = decltype(token)::value;
                            e[t] = score[i][t] * of_lane<t>(vs[i][m]);
                        });
                        if (masked) {           // what is not seen may have any scale
                            asm volatile("" : "+v"(from[i]), "+v"(count[i]));       // compared again, not kept
#pragma unroll
                            for (int t = 0; t < 16; ++t) e[t] = (uint32_t)(t - from[i]) < count[i] ? e[t] : 0.0f;
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) split_in_two(e + 8 * j, p[2 * i + j], rest[2 * i + j]);
                    });
                    // no product after one on the same sums, where there are others
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        bf16x8 v[kPer];
#pragma unroll
                        for (int t = 0; t < kPer; ++t) {
                            v[t] = *reinterpret_cast<const bf16x8 *>(tile + RowsTile<D, NB>::kKeys + ((m * kPer + t) * 4 + i) * 1024 + lane * 16);
                            o[m * kPer + t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[t], p[i], o[m * kPer + t], 0, 0, 0);
                        }
#pragma unroll
                        for (int t = 0; t < kPer; ++t)
                            o[m * kPer + t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[t], rest[i], o[m * kPer + t], 0, 0, 0);
                    }
                });
            }
            cur ^= 1;
            if (t0 + 64 < span.last) next.store(lds[cur], call.scale, wave, lane);
        }
        total = halves_sum(total);
        if (row0 + r >= rows) continue;
        const int64_t place_out = place_of_row(call, q0, row);
        if (call.splits == 1) {
            const float inverse = ends_with(base, total);
#pragma unroll
            for (int t = 0; t < D / 32; ++t) {
                const v16f done = o[t] * inverse;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<u32x2 *>(call.out + place_out * D + t * 32 + 8 * j + 4 * half) =
                        u32x2{narrow_bf16x2(done[4 * j], done[4 * j + 1]), narrow_bf16x2(done[4 * j + 2], done[4 * j + 3])};
            }
            if (call.lse && half == 0) call.lse[place_out] = log_sum(base, total);
        } else {
            const int64_t all = call.q_rows * call.q_heads, part = split * all + place_out;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<v4f *>(call.part + part * D + t * 32 + 8 * j + 4 * half) =
                        v4f{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
            if (half == 0) reinterpret_cast<float2 *>(call.part + call.splits * all * D)[part] = float2{base, total};
        }
    }
}

// ---- few rows of short sequences: the waves of a workgroup have the same ones and different tokens
// Grid: tiles of rows, heads, sequences.

template <int D, int NB, int R>
__global__ __launch_bounds__(256) void attention_tokens_kernel(const AttentionCall call, const Sequences seqs, const Pool pool)
{
    constexpr int kRows = R * 16, kPitch = D + 4;           // of a row of results in LDS, whose statistics are behind it
    __shared__ float joined[2][kRows][kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int b = blockIdx.z, h = blockIdx.y;
    const int q0 = within(call.q_starts[b], call.q_rows), queries = within(call.q_starts[b + 1], call.q_rows) - q0;
    const int length = seqs.length(b, pool.page);
    const int rows = queries * call.group, tiles = (rows + kRows - 1) / kRows;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int row0 = tile * kRows;
        Rows<D, NB, R> mine;
        load_q(mine, call, q0, queries, h, row0, lane);
        start_rows(mine, call, queries, length, h, row0, lane);
        const Span span = span_of(call, queries, length, row0, row0 + kRows - 1);
        walk<256>(mine, pool, seqs.table + b * seqs.width, seqs.width, h, call.scale, span.first + wave * 64, span.last, span, lane);
#pragma unroll
        for (int n = 0; n < R; ++n) mine.total[n] = quarters_sum(mine.total[n]);
        // join the four waves: two halves, then one
        auto give = [&](int half) {
#pragma unroll
            for (int n = 0; n < R; ++n) {
                float *const row = joined[half][n * 16 + r];
#pragma unroll
                for (int t = 0; t < D / 16; ++t) *reinterpret_cast<v4f *>(row + t * 16 + 4 * g) = mine.o[n][t];
                if (g == 0) {
                    row[D] = mine.base[n];
                    row[D + 1] = mine.total[n];
                }
            }
        };
        auto take = [&](int half) {
#pragma unroll
            for (int n = 0; n < R; ++n) {
                const float *const row = joined[half][n * 16 + r];
                const float base = row[D], now = __builtin_fmaxf(mine.base[n], base);
                const float reference = now == -__builtin_inff() ? 0.0f : now;
                const float fade = __builtin_amdgcn_exp2f(mine.base[n] - reference), other = __builtin_amdgcn_exp2f(base - reference);
                mine.base[n] = now;
                mine.total[n] = mine.total[n] * fade + row[D + 1] * other;
#pragma unroll
                for (int t = 0; t < D / 16; ++t)
                    mine.o[n][t] = mine.o[n][t] * fade + *reinterpret_cast<const v4f *>(row + t * 16 + 4 * g) * other;
            }
        };
        __syncthreads();                // the last rows' results have been read
        if (wave >= 2) give(wave - 2);
        __syncthreads();
        if (wave < 2) take(wave);
        __syncthreads();
        if (wave == 1) give(0);
        __syncthreads();
        if (wave != 0) continue;
        take(0);
#pragma unroll
        for (int n = 0; n < R; ++n) {
            if (row0 + n * 16 + r < rows) end_row(mine, n, call, place_of_row(call, q0, Row(call, queries, h, row0 + n * 16 + r)), lane);
        }
    }
}

// ---- few rows of any sequences: every wave has an even share of all that is to be done
// What is to be done is counted in tiles of 64 tokens for one tile of rows and key head (an item).  Wave w has the tiles w * per ..
// (w + 1) * per - 1 of all sequences' items in order and walks through them without a pause, asking for an item's first tile
// while it ends the one before (with a workgroup an item and sequence, the longest took as long again as all together; with shares
// of workgroups that began every item anew, an item's beginning took as long as 500 tokens).  The part of an item that it
// has, if not the whole, goes to its slot 0 where the item began before, to slot 1 where it begins here; the join finds the
// parts by the same count.

constexpr int kShares = 2048;               // waves: eight a CU
constexpr int kMostShared = 1024;           // sequences that a workgroup counts

// What a workgroup knows of the sequences: before[b] tiles are of those before b, before[count] of all.
struct Counted {
    int64_t before[kMostShared + 1], wave_sums[4];
    int q0[kMostShared + 1], length[kMostShared];
};

// An item's tiles, and where they begin.
struct ItemTiles {
    int first, tiles;
    __device__ __forceinline__ ItemTiles(const AttentionCall &call, int queries, int length)
    {
        first = queries <= 0 ? 0 : span_of(call, queries, length, 0, 0).first;
        tiles = length > first ? (length - first + 63) / 64 : 1;
    }
};

// The whole workgroup.
__device__ __forceinline__ void count_tiles(Counted &all, const AttentionCall &call, const Sequences &seqs, const Pool &pool, int tile_rows)
{
    constexpr int kPer = kMostShared / 256;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t mine[kPer], sum = 0;
    const int per = (call.sequences + 255) / 256;           // of a thread: one up to 256 sequences
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = threadIdx.x * per + i;
        mine[i] = 0;
        if (i < per && b < call.sequences) {
            const int q0 = within(call.q_starts[b], call.q_rows), past = within(call.q_starts[b + 1], call.q_rows);
            const int length = seqs.length(b, pool.page);
            all.q0[b] = q0;
            if (b + 1 == call.sequences) all.q0[b + 1] = past;
            all.length[b] = length;
            if (past > q0) {
                const int items = ((past - q0) * call.group + tile_rows - 1) / tile_rows * pool.heads;
                mine[i] = (int64_t)items * ItemTiles(call, past - q0, length).tiles;
            }
        }
        sum += mine[i];
    }
    int64_t upto = sum;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const int64_t other = __shfl_up(upto, step);
        if (lane >= step) upto += other;
    }
    if (lane == 63) all.wave_sums[wave] = upto;
    __syncthreads();
    int64_t at = upto - sum;
    for (int i = 0; i < wave; ++i) at += all.wave_sums[i];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = threadIdx.x * per + i;
        if (i < per && b <= call.sequences) all.before[b] = at;
        at += mine[i];
    }
    if (call.sequences == per * 256 && threadIdx.x == 255) all.before[call.sequences] = at;
    __syncthreads();
}

// The tiles of a share: up to two, eight waves a CU have them; more are shared out among four, which ask for as much at a time as
// the memory gives, and leave fewer parts (MI355X, 30 thousand tiles: 93 us against 99; 1100 tiles in eight 12.4, in four 19.8).
__host__ __device__ inline int64_t share_of(int64_t tiles)
{
    const int64_t per = (tiles + kShares - 1) / kShares;
    return per <= 2 ? per : (tiles + kShares / 2 - 1) / (kShares / 2);
}

// What the join needs of the count: before[], behind the parts' statistics.
template <int D, int R>
__device__ __forceinline__ int64_t *kept_count(const AttentionCall &call)
{
    return reinterpret_cast<int64_t *>(call.part + (int64_t)kShares * 2 * R * 16 * (D + 2));
}

// Slot `slot` of wave w: its row's place among the parts.
template <int R>
__device__ __forceinline__ int64_t slot_row(int w, int slot, int row) { return ((int64_t)w * 2 + slot) * (R * 16) + row; }
template <int D, int R>
__device__ __forceinline__ float2 *slot_stats(const AttentionCall &call)
{
    return reinterpret_cast<float2 *>(call.part + (int64_t)kShares * 2 * R * 16 * D);
}

// A place in a wave's walk: an item and a tile of it; all the same in every lane.
struct Cursor {
    int b, h, row0, t;          // sequence, key head, first row; first token of the tile
    int q0, queries, length, first, last;       // of the sequence; tokens first .. last - 1 are the item's

    __device__ __forceinline__ void enter(const Counted &all, const AttentionCall &call, int sequence)
    {
        b = __builtin_amdgcn_readfirstlane(sequence);
        q0 = __builtin_amdgcn_readfirstlane(all.q0[b]);
        queries = __builtin_amdgcn_readfirstlane(all.q0[b + 1]) - q0;
        length = __builtin_amdgcn_readfirstlane(all.length[b]);
        const ItemTiles item(call, queries, length);
        first = item.first;
        last = item.first + item.tiles * 64;
    }
    // The next tile; past the last item of all, one that is loaded and not used.
    __device__ __forceinline__ void advance(const Counted &all, const AttentionCall &call, const Pool &pool, int tile_rows)
    {
        t += 64;
        if (t < last) return;
        t = first;
        if (++h < pool.heads) return;
        h = 0;
        row0 += tile_rows;
        if (row0 < queries * call.group) return;
        row0 = 0;
        int next = b + 1;
        while (next < call.sequences && all.q0[next + 1] <= all.q0[next]) ++next;       // without queries: no items
        if (next >= call.sequences) return;
        enter(all, call, next);
        t = first;
    }
};

template <int D, int NB, int R>
__global__ __launch_bounds__(256, R == 1 && D <= 128 ? 2 : 1) void attention_shares_kernel(const AttentionCall call,
                                                                                           const Sequences seqs, const Pool pool)
{
    constexpr int kRows = R * 16;
    __shared__ Counted all;
    const int lane = threadIdx.x & 63, share = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int r = lane & 15, g = lane >> 4;
    count_tiles(all, call, seqs, pool, kRows);
    const int64_t total = all.before[call.sequences], per = share_of(total), from = share * per;
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b <= call.sequences; b += 256) kept_count<D, R>(call)[b] = all.before[b];
    }
    if (from >= total) return;
    int left = __builtin_amdgcn_readfirstlane((int)(total - from < per ? total - from : per));
    Cursor at;                          // what is computed
    {
        int b = 0, past = call.sequences;       // before[b] <= from < before[past]
        while (past - b > 1) {
            const int middle = (b + past) / 2;
            if (all.before[middle] <= from) {
                b = middle;
            } else {
                past = middle;
            }
        }
        at.enter(all, call, b);
        const int64_t mine = from - all.before[b];
        const int tiles = (at.last - at.first) / 64;
        const int item = __builtin_amdgcn_readfirstlane((int)(mine / tiles));
        at.t = at.first + __builtin_amdgcn_readfirstlane((int)(mine - (int64_t)item * tiles)) * 64;
        const int row_tile = item / pool.heads;
        at.h = item - row_tile * pool.heads;
        at.row0 = row_tile * kRows;
    }
    auto ids_of = [&](const Cursor &c) { return PageIds(pool, seqs.table + c.b * seqs.width, seqs.width, c.t, lane); };
    Rows<D, NB, R> mine;
    Tile<D, NB> tile;
    load_q(mine, call, at.q0, at.queries, at.h, at.row0, lane);
    bool there;
    {
        const Place place(pool, ids_of(at), at.h, at.t, lane);
        tile.load_k(pool, place.k_at, place.k_in, place.v_at, place.v_in, lane);
        tile.load_v(pool, place.v_at, place.v_in, lane);
        there = place.there;
    }
    Cursor next = at;                   // what is loaded
    next.advance(all, call, pool, kRows);
    PageIds ids = ids_of(next);
    start_rows(mine, call, at.queries, at.length, at.h, at.row0, lane);
    Span span = span_of(call, at.queries, at.length, at.row0, at.row0 + kRows - 1);
    bool begun_here = at.t == at.first;
    for (;;) {
        const Place place(pool, ids, next.h, next.t, lane);
        float score[R][16];
        mine.scores(tile, call.scale, score);
        tile.load_k(pool, place.k_at, place.k_in, place.v_at, place.v_in, lane);
        const bool item_ends = at.t + 64 >= at.last, ends = item_ends || left == 1;
        if (ends) load_q(mine, call, next.q0, next.queries, next.h, next.row0, lane);
        Cursor after = next;
        after.advance(all, call, pool, kRows);
        ids = ids_of(after);
        __builtin_amdgcn_sched_barrier(0);
        mine.add(tile, score, at.t + 16 * g, there, !(at.t >= span.all_from && at.t + 64 <= span.all_to && __all(there)));
        tile.load_v(pool, place.v_at, place.v_in, lane);
        there = place.there;
        if (ends) {
#pragma unroll
            for (int n = 0; n < R; ++n) {
                mine.total[n] = quarters_sum(mine.total[n]);
                const int row = at.row0 + n * 16 + r;
                if (row >= at.queries * call.group) continue;
                if (begun_here && item_ends) {
                    end_row(mine, n, call, place_of_row(call, at.q0, Row(call, at.queries, at.h, row)), lane);
                } else {
                    const int64_t place_in = slot_row<R>(share, begun_here ? 1 : 0, n * 16 + r);
                    part_row(mine, n, call.part + place_in * D, slot_stats<D, R>(call) + place_in, lane);
                }
            }
            if (left == 1) return;
            start_rows(mine, call, next.queries, next.length, next.h, next.row0, lane);
            span = span_of(call, next.queries, next.length, next.row0, next.row0 + kRows - 1);
            begun_here = true;
        }
        --left;
        at = next;
        next = after;
    }
}

// ---- joining parts
// An output row and head has W of a workgroup's four waves, which take 64 parts each at a time; in a wave D / 4 lanes take a part, the
// others other parts, and the sums are added in order.  Little is read and much waited for: what can be asked for at once is (one
// part's statistics after the other's: 17.5 us for 64).

template <int D, int W>
struct Joiner {
    static constexpr int kLanes = D / 4, kParts = 64 / kLanes, kRounds = 64 / kParts < 8 ? 64 / kParts : 8;
    struct Shared {
        v4f acc[256];
        float2 stats[4];
    };
    float now = -__builtin_inff(), total = 0.0f;
    v4f acc = {0, 0, 0, 0};

    // `count` parts: part i's statistics are at stat_of(i), its sums at sums_of(i)
    template <typename Stat, typename Sums>
    __device__ __forceinline__ void join(int count, Stat stat_of, Sums sums_of)
    {
        const int thread = threadIdx.x & 63, mine = thread / kLanes, lane = thread % kLanes;
        for (int at = threadIdx.x % (W * 64) / 64 * 64; at < count; at += W * 64) {
            const float2 stat = at + thread < count ? *stat_of(at + thread) : float2{-__builtin_inff(), 0.0f};
            v4f o[kRounds];
            auto load = [&](int from) {
#pragma unroll
                for (int i = 0; i < kRounds; ++i) {
                    const int p = at + from + mine + i * kParts;
                    o[i] = p < count ? *reinterpret_cast<const v4f *>(sums_of(p) + lane * 4) : v4f{0, 0, 0, 0};
                }
            };
            load(0);
            loads_first();
            float most = __builtin_fmaxf(stat.x, now);
#pragma unroll
            for (int step = 1; step < 64; step *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, step));
            const float reference = most == -__builtin_inff() ? 0.0f : most;
            const float weight = __builtin_amdgcn_exp2f(stat.x - reference), fade = __builtin_amdgcn_exp2f(now - reference);
            float sum = stat.y * weight;
#pragma unroll
            for (int step = 1; step < 64; step *= 2) sum += __shfl_xor(sum, step);
            total = total * fade + sum;
            acc *= fade;
            now = most;
            for (int from = 0;;) {
#pragma unroll
                for (int i = 0; i < kRounds; ++i) acc += o[i] * __shfl(weight, (from + mine + i * kParts) & 63);
                from += kRounds * kParts;
                if (from >= 64 || at + from >= count) break;
                load(from);
            }
        }
    }
    // The whole workgroup, rows that have nothing to join among it.
    __device__ __forceinline__ void end(Shared &shared, const AttentionCall &call, int64_t at, bool write)
    {
        const int thread = threadIdx.x % (W * 64), wave = threadIdx.x / 64, first = wave / W * W;
        shared.acc[threadIdx.x] = acc;
        if (threadIdx.x % 64 == 0) shared.stats[wave] = float2{now, total};
        __syncthreads();
        if (!write || thread >= kLanes) return;
        float most = shared.stats[first].x;
#pragma unroll
        for (int w = 1; w < W; ++w) most = __builtin_fmaxf(most, shared.stats[first + w].x);
        const float reference = most == -__builtin_inff() ? 0.0f : most;
        acc = v4f{0, 0, 0, 0};
        total = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float weight = __builtin_amdgcn_exp2f(shared.stats[first + w].x - reference);
            total += shared.stats[first + w].y * weight;
#pragma unroll
            for (int p = 0; p < kParts; ++p) acc += shared.acc[(first + w) * 64 + p * kLanes + thread] * weight;
        }
        acc *= ends_with(most, total);
        *reinterpret_cast<u32x2 *>(call.out + at * D + thread * 4) = u32x2{narrow_bf16x2(acc[0], acc[1]), narrow_bf16x2(acc[2], acc[3])};
        if (call.lse && thread == 0) call.lse[at] = log_sum(most, total);
    }
};

// The splits of attention_rows_kernel, for output rows and heads from `first` on.
template <int D, int W>
__global__ __launch_bounds__(256) void join_splits_kernel(const AttentionCall call, int64_t first)
{
    __shared__ typename Joiner<D, W>::Shared shared;
    const int64_t all = call.q_rows * call.q_heads, at = first + (int64_t)blockIdx.x * (4 / W) + threadIdx.x / (W * 64);
    const int row = (int)((uint32_t)at / (uint32_t)call.q_heads);
    const bool write = at < all && row >= call.q_starts[0] && row < call.q_starts[call.sequences];     // not a row of no sequence
    Joiner<D, W> joiner;
    const float2 *const stats = reinterpret_cast<const float2 *>(call.part + call.splits * all * D) + at;
    joiner.join(write ? call.splits : 0, [&](int s) { return stats + s * all; },
                [&](int s) { return call.part + (s * all + at) * D; });
    joiner.end(shared, call, at, write);
}

// The shares of attention_shares_kernel, where a row's item is of more than one: otherwise the wave that had it wrote it.
template <int D, int R, int W>
__global__ __launch_bounds__(256) void join_shares_kernel(const AttentionCall call, const Sequences seqs, const Pool pool,
                                                          int64_t first_row)
{
    __shared__ typename Joiner<D, W>::Shared shared;
    const int lane = threadIdx.x & 63;
    const int64_t at = first_row + (int64_t)blockIdx.x * (4 / W) + threadIdx.x / (W * 64);
    const int row = (int)((uint32_t)at / (uint32_t)call.q_heads), head = (int)at - row * call.q_heads;
    // the row's sequence, by the wave: the last one that begins with it or before, and has it
    int b = -1;
    for (int from = 0; from < call.sequences; from += 64) {
        const int i = from + lane < call.sequences ? from + lane : call.sequences - 1;
        const uint64_t has = __ballot(row >= call.q_starts[i] && row < call.q_starts[i + 1] && at < call.q_rows * call.q_heads);
        if (has) b = from + __builtin_ctzll(has);
    }
    if (b >= call.sequences) b = call.sequences - 1;
    int count = 0, first = 0, mine = 0;
    if (b >= 0) {
        const int64_t *const before = kept_count<D, R>(call);
        const int q0 = within(call.q_starts[b], call.q_rows), queries = within(call.q_starts[b + 1], call.q_rows) - q0;
        const int tiles = ItemTiles(call, queries, seqs.length(b, pool.page)).tiles;
        const int64_t per = share_of(before[call.sequences]);
        const int h = head / call.group;
        mine = (row - q0) * call.group + head - h * call.group;
        const int64_t from = before[b] + ((int64_t)(mine / (R * 16)) * pool.heads + h) * tiles;
        first = (int)(from / per);
        count = (int)((from + tiles - 1) / per) - first + 1;
        if (count == 1) count = 0;
    }
    Joiner<D, W> joiner;
    auto place = [&](int p) { return slot_row<R>(first + p, p == 0 ? 1 : 0, mine % (R * 16)); };
    joiner.join(count, [&](int p) { return slot_stats<D, R>(call) + place(p); }, [&](int p) { return call.part + place(p) * D; });
    joiner.end(shared, call, at, count > 0);
}

}  // namespace cache
}  // namespace equarx
