// Device code of the 4-bit microscaled format: quantizing rows, reading them back, and the product of packed rows.
#pragma once

#include <type_traits>
#include <utility>

#include "equarx_rows.hpp"

namespace equarx {
namespace mx4 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------- one block's scale and codes

// The larger of each half of two words, as unsigned 16-bit numbers: magnitudes of bf16 numbers are ordered like their
// patterns.
__device__ __forceinline__ uint32_t umax16x2(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Eight bf16 numbers as codes at a scale: the hardware rounds to nearest, ties to even, and clamps at 6.
__device__ __forceinline__ uint32_t codes_of(const u32x4 &x, float scale)
{
    const uint32_t d[4] = {x.x, x.y, x.z, x.w};      // not a cast of x[i]: the compiler casts the first element each time
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, d[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, d[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, d[2]), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, d[3]), scale, 3);
    return w;
}

__device__ __forceinline__ uint32_t magnitudes_max(const u32x4 &x)
{
    constexpr uint32_t kMagnitude = 0x7fff7fffu;
    return umax16x2(umax16x2(x[0] & kMagnitude, x[1] & kMagnitude), umax16x2(x[2] & kMagnitude, x[3] & kMagnitude));
}

// Eight elements of a block as codes, with the block's scale byte; the other 24 are in the other lanes of the quad.
__device__ __forceinline__ uint32_t pack_unit(const u32x4 &v, uint32_t &byte)
{
    uint32_t top = magnitudes_max(v);
    top = umax(top & 0xffff, top >> 16);
    top = umax(top, dpp_read<0xB1>(top));
    top = umax(top, dpp_read<0x4E>(top));
    byte = scale_byte(top);
    return byte == 255 ? 0 : codes_of(v, scale_of(byte));
}

// ---------------------------------------------------------------- rows <-> packed rows
// A lane has eight elements, a quad a block, a row of sixteen lanes a group: `units` pieces of eight in all, the
// padding among them, `unit` counting through the packed rows.  Memory is the bound: 4096 x 5376 in 10.2 us either way, 5.5 TB/s.

__global__ __launch_bounds__(256) void quantize_rows_kernel(Global<const uint16_t> x, int64_t x_stride, Global<uint8_t> codes,
                                                            Global<uint8_t> scales, int64_t cols, uint32_t units,
                                                            const Divisor row_units)
{
    const uint32_t unit = blockIdx.x * 256 + threadIdx.x;
    if (unit >= units) return;                                  // whole rows of sixteen lanes: units is a multiple of 16
    const uint32_t row = row_units.of(unit);
    const int64_t col = (int64_t)(unit - row * row_units.d) * 8;
    uint32_t byte;
    const u32x4 v = load_row8(x + row * x_stride, col, cols);
    reinterpret_cast<uint32_t *>((uint8_t *)codes)[unit] = pack_unit(v, byte);
    uint32_t four = byte << (8 * ((threadIdx.x >> 2) & 3));
    four |= dpp_read<0x141>(four);
    four |= dpp_read<0x140>(four);
    if ((threadIdx.x & 15) == 0) reinterpret_cast<uint32_t *>((uint8_t *)scales)[unit / 16] = four;
}

__device__ __forceinline__ u32x4 values_of(uint32_t codes, float scale)
{
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return v;
}

__global__ __launch_bounds__(256) void dequantize_rows_kernel(Global<const uint8_t> codes, Global<const uint8_t> scales,
                                                              Global<uint16_t> out, int64_t out_stride, int64_t cols,
                                                              uint32_t units, const Divisor row_units)
{
    const uint32_t unit = blockIdx.x * 256 + threadIdx.x;
    if (unit >= units) return;
    const uint32_t row = row_units.of(unit);
    const int64_t col = (int64_t)(unit - row * row_units.d) * 8;
    if (col >= cols) return;
    const uint32_t w = reinterpret_cast<const uint32_t *>((const uint8_t *)codes)[unit];
    const uint32_t byte = scales[unit / 4];
    u32x4 v = values_of(w, scale_of(byte));
    if (byte == 255) v = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    store_row8(out + row * out_stride, col, cols, v);
}

// ---------------------------------------------------------------- product of packed rows
// With the operands as w (rows of the result) and x (its columns) one 32x32x64 instruction takes two blocks of 32 rows of w and of 32
// rows of x: lane l has row l % 32 and one of the two, l / 32, with the block's scale, any byte of a register.  Its result
// lane l has column l % 32, a row of x, and the rows of w 8 q + 4 (l / 32) + 0 .. 3, q = 0 .. 3: four consecutive outputs each.

template <int kScaleByte>
__device__ __forceinline__ v16f multiply(const u32x4 &w, uint32_t w_scale, const u32x4 &x, uint32_t x_scale, const v16f &sum)
{
    const v8i a = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    const v8i b = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sum, 4, 4, kScaleByte, (int)w_scale, kScaleByte, (int)x_scale);
}

// Four consecutive outputs of one row, as far as the row goes.
__device__ __forceinline__ void store_out4(uint16_t *row, int64_t n, int64_t N, const v4f &v)
{
    typedef u32x2 u32x2_anywhere __attribute__((aligned(2)));
    const u32x2 w = {narrow_bf16x2(v[0], v[1]), narrow_bf16x2(v[2], v[3])};
    if (n + 4 <= N) {
        *reinterpret_cast<u32x2_anywhere *>(row + n) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i < N) row[n + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
}

// One direct load of 16 bytes a lane: LDS `to` + lane * 16 <- `from` + `offset`.
__device__ __forceinline__ void direct_load(uint32_t to, const uint8_t *from, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}

__device__ __forceinline__ void direct_load(uint32_t to, const uint8_t *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}

// A lane's 32-bit offset reaches 256 rows of codes of the longest product there is.
constexpr int64_t kMostK = (int64_t)1 << 24;

// ---- few rows of x
// A workgroup has 32 rows of w and MT * 32 rows of x, and walks over all of k; what bounds it is reading w once, so what counts is
// bytes in flight.  Pairs of groups, 128 bytes of every row, come to LDS with direct loads, kDepth - 1 pairs ahead of their turn (a lane
// that loads its row's bytes into registers itself has its neighbours on other lines: 64 rows of x by 5376 x 5376 15.4 us; this way
// 10.2 with the packing of x, two launches of 2.1 us that do nothing among them, and one row by 5376 x 4096 6.0 us).  With N / 32
// workgroups, 168 of these, 88 of the 256 CUs have none.
// In a pair wave q of the four has the blocks 2 q and 2 q + 1 of all rows, one instruction for 32 rows of x; the waves' sums are added
// in order at the end.  LDS: a row is its 128 bytes, block b of row r in place b xor r / 2 % 8, which spreads sixteen rows' block
// over all banks; of scales four groups' 16 bytes a row, every second pair.
//
// kQuantize: x is bf16 and little; every workgroup packs all of it into LDS first, with its first rows of w on the way.

constexpr int kMostQuantized = 1 << 15;             // elements of x that a workgroup packs itself, padded groups counted
constexpr int kMostQuantizedRows = 32;

template <int MT, bool kQuantize>
__global__ __launch_bounds__(256) void product_rows_kernel(Global<const uint8_t> xc, Global<const uint8_t> xs,
                                                           Global<const uint8_t> wc, Global<const uint8_t> ws, Global<uint16_t> out,
                                                           int32_t M, int32_t N, int32_t groups, int64_t out_stride,
                                                           int64_t x_stride, int32_t K)
{
    constexpr int W = 4, kSides = kQuantize ? 1 : 1 + MT;           // of 32 rows each, w first
    constexpr int kDepth = MT == 4 ? 6 : 8;
    constexpr int kPair = kSides * 4096, kScales = (kSides * 512 + 1023) / 1024 * 1024;     // bytes of codes; of four groups' scales
    constexpr int kWindows = kDepth / 2 + 1;                        // fours of groups that the pairs in flight are of
    constexpr int kScalesAt = kDepth * kPair, kXAt = kScalesAt + kWindows * kScales;
    constexpr int kPacked = kQuantize ? kMostQuantized / 2 + kMostQuantized / 32 + kMostQuantizedRows * 16 : 0;
    constexpr int kAll = kXAt + kPacked, kParts = W * MT * 4096;
    static_assert(kDepth % 2 == 0 && (!kQuantize || MT == 1), "fours are of two pairs; little is a tile's rows");
    __shared__ __align__(1024) uint8_t lds[kAll > kParts ? kAll : kParts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5;
    const int64_t n0 = (int64_t)blockIdx.x * 32, m0 = (int64_t)blockIdx.y * (32 * MT);
    const int64_t blocks = (int64_t)groups * 4;
    const int pairs = (groups + 1) / 2;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

    // x that is packed here: what a thread reads first is asked for before w
    constexpr int kFirst = 4;
    const int row_units = groups * 16, units = kQuantize ? M * row_units : 0, x_pitch = groups * 64 + 16;
    u32x4 unit_of_x[kFirst];
    auto load_unit = [&](int unit) {
        const int row = unit / row_units, col = (unit - row * row_units) * 8;
        return load_row8(reinterpret_cast<const uint16_t *>((const uint8_t *)xc) + row * x_stride, col, K);
    };
    auto pack = [&](int unit, const u32x4 &v) {                     // whole rows of sixteen lanes together
        const int row = unit / row_units, at = unit - row * row_units;
        uint32_t byte;
        const uint32_t codes = pack_unit(v, byte);
        *reinterpret_cast<uint32_t *>(lds + kXAt + row * x_pitch + at * 4) = codes;
        if (unit % 4 == 0) lds[kXAt + M * x_pitch + unit / 4] = (uint8_t)byte;
    };
    if constexpr (kQuantize) {
#pragma unroll
        for (int i = 0; i < kFirst; ++i) {
            const int unit = threadIdx.x + i * 64 * W;
            unit_of_x[i] = unit < units ? load_unit(unit) : u32x4{0, 0, 0, 0};
        }
    }

    // Loads: eight rows of a side are one, wave q has rows 8 q .. 8 q + 7 of every side; of scales it is 64 rows of all sides.
    const uint8_t *code_from[kSides];
    uint32_t code_at[kSides];
    const int eight = wave * 8 + lane / 8, block = (lane & 7) ^ (eight >> 1 & 7);
    auto row_of = [&](int side, int i) {                            // past the end the last row again, stored nowhere
        const int64_t row = (side == 0 ? n0 : m0 + 32 * (side - 1)) + i, most = (side == 0 ? N : M) - 1;
        return row < most ? row : most;
    };
#pragma unroll
    for (int i = 0; i < kSides; ++i) {
        code_from[i] = (i == 0 ? (const uint8_t *)wc : (const uint8_t *)xc) + row_of(i, 0) * blocks * 16;
        code_at[i] = (uint32_t)((row_of(i, eight) - row_of(i, 0)) * blocks * 16) + block * 16;
    }
    const bool has_scales = wave * 64 < kSides * 32 && groups >= 4;
    const int scale_side = wave * 2 + h < kSides ? wave * 2 + h : kSides - 1;
    const uint8_t *const scale_from = (scale_side == 0 ? (const uint8_t *)ws : (const uint8_t *)xs) + row_of(scale_side, r) * blocks;
    // the four groups of scales that a pair's belong to; the last four of a row may begin inside the four before
    auto window = [&](int pair) { return groups < 4 ? 0 : pair / 2 * 4 + 4 <= groups ? pair / 2 * 4 : groups - 4; };
    auto issue = [&](int pair, int slot_at, bool even) {            // past the end the last pair again, not used
        const int p = pair < pairs ? pair : pairs - 1;
        if (even && has_scales)
            direct_load(base + kScalesAt + (uint32_t)(pair / 2 % kWindows) * kScales + wave * 1024, scale_from + window(p) * 4);
        const uint32_t second = 2 * p + 1 == groups && block >= 4 ? 64 : 0;     // the last group is alone: it stands in
#pragma unroll
        for (int i = 0; i < kSides; ++i)
            direct_load(base + slot_at + i * 4096 + wave * 1024, code_from[i] + (int64_t)p * 128, code_at[i] - second);
    };
    if (groups < 4) {                                               // too few for a load of four
        for (int i = threadIdx.x; i < kSides * 32; i += 64 * W) {
            const uint8_t *const from = (i < 32 ? (const uint8_t *)ws : (const uint8_t *)xs) + row_of(i / 32, i % 32) * blocks;
            for (int g = 0; g < groups; ++g)
                *reinterpret_cast<uint32_t *>(lds + kScalesAt + i * 16 + g * 4) = *reinterpret_cast<const uint32_t *>(from + g * 4);
        }
    }
    if (groups > 0) {
#pragma unroll
        for (int i = 0; i < kDepth - 1; ++i) issue(i, i * kPair, i % 2 == 0);
    }
    if constexpr (kQuantize) {
#pragma unroll
        for (int i = 0; i < kFirst; ++i) {
            const int unit = threadIdx.x + i * 64 * W;
            if (unit < units) pack(unit, unit_of_x[i]);
        }
        for (int unit = threadIdx.x + kFirst * 64 * W; unit < units; unit += 64 * W) pack(unit, load_unit(unit));
    }
    v16f sum[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) sum[t] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const int mine = 2 * wave + h, place = r * 128 + (mine ^ (r >> 1 & 7)) * 16;    // this lane's block of a pair, where it lies
    const int x_row = r < M ? r : M - 1;
    struct Fragment {
        u32x4 w, x[MT];
        uint32_t w_scale, x_scale[MT];
    } f[2];
    auto read = [&](Fragment &to, int pair, int slot_at) {
        const uint8_t *const codes = lds + slot_at + place;
        const int group = (2 * pair + wave / 2 - window(pair)) & 3;
        const uint8_t *const scales = lds + kScalesAt + (uint32_t)(pair / 2 % kWindows) * kScales + r * 16 + group * 4 + (mine & 3);
        to.w = *reinterpret_cast<const u32x4 *>(codes);
        to.w_scale = *scales;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if constexpr (kQuantize) {
                const int at = pair < pairs ? pair * 8 + mine : mine;
                to.x[t] = *reinterpret_cast<const u32x4 *>(lds + kXAt + x_row * x_pitch + at * 16);
                to.x_scale[t] = lds[kXAt + M * x_pitch + x_row * (int)blocks + at];
            } else {
                to.x[t] = *reinterpret_cast<const u32x4 *>(codes + (t + 1) * 4096);
                to.x_scale[t] = scales[(t + 1) * 512];
            }
        }
    };
    auto multiply_all = [&](Fragment &f) {
#pragma unroll
        for (int t = 0; t < MT; ++t) sum[t] = multiply<0>(f.w, f.w_scale, f.x[t], f.x_scale[t], sum[t]);
    };
    // Turn by turn: the next pair is in LDS for all waves, and this one in registers; the one before has been read by all, its
    // buffer is free.
    auto after = [](int slot_at) { return slot_at + kPair == kDepth * kPair ? 0 : slot_at + kPair; };
    int slot_at = 0, next_at = (kDepth - 1) * kPair;
    auto turn = [&](int pair, int now) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kDepth - 3) * kSides) : "memory");
        slot_at = after(slot_at);
        issue(pair + kDepth - 1, next_at, (kDepth - 1 + now) % 2 == 0);
        next_at = after(next_at);
        read(f[1 - now], pair + 1, slot_at);
        multiply_all(f[now]);
    };
    if (groups > 0) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kDepth - 2) * kSides) : "memory");
        read(f[0], 0, 0);
        // the last pair is left over: a group that is alone has blocks for two of the waves
        int pair = 0;
        for (; pair + 2 < pairs; pair += 2) {
            turn(pair, 0);
            turn(pair + 1, 1);
        }
        if (pair + 1 < pairs) {
            turn(pair, 0);
            f[0] = f[1];
        }
        if (2 * pairs == groups || wave < 2) multiply_all(f[0]);
    }
    // what was loaded past the end has landed, and all have read: LDS takes the waves' sums
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    v4f *const part = reinterpret_cast<v4f *>(lds);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            part[((wave * MT + t) * 4 + q) * 64 + lane] = v4f{sum[t][4 * q], sum[t][4 * q + 1], sum[t][4 * q + 2], sum[t][4 * q + 3]};
    __syncthreads();
    for (int i = wave; i < MT * 4; i += W) {
        v4f total = part[i * 64 + lane];
#pragma unroll
        for (int p = 1; p < W; ++p) total += part[(p * MT * 4 + i) * 64 + lane];
        const int64_t m = m0 + 32 * (i / 4) + r;
        if (m < M) store_out4(out + m * out_stride, n0 + 8 * (i % 4) + 4 * h, N, total);
    }
}

// ---- large products
// A workgroup of WN x WM waves has WN * FN * 32 rows of w by WM * FM * 32 rows of x, a wave FN x FM results of 32 x 32 in
// registers.  A step is the 128 elements of a group, two 32x32x64 instructions a result, whose lane l has row l % 32 and block l / 32
// of two.  Codes come to LDS with direct loads of two steps, a pair, into one of kBuffers buffers: a pair is asked for when
// the one kBuffers before it has been read.
//
// In LDS a row of a pair is 128 bytes, a line of memory, and rows follow each other as the lanes of a direct load do, eight
// lanes a row (rows spread over distant lanes, or half lines, are more requests: 8192 cubed 383 and 291 us).  The eight blocks of
// row r stand in the order of their number xor r / 2 % 8, so that one block of sixteen rows is in all banks once (a third of the LDS
// cycles are counted as conflicts all the same; the words of scales, 16 bytes apart, are a sixth of those at most).  Scales: the
// four bytes of a row and step are a word; a lane shifts it by its block and the instruction picks byte 0 or 2.  Rows' scales lie
// far apart, a line each, so that they are loaded for four steps at once (a word a step: half of all requests).
//
// 8192 cubed: 274 us, 4.0 PFLOP/s, where the instruction alone on such operands does 6.6 with the clock that the power leaves it; the
// matrix unit is busy for 56 to 57 % of the cycles, the rest are the codes' way to LDS, which takes about as long as they, and 30 us
// of results on their way out that nothing runs beside.

// What one of W waves loads of a side: of every pair eights of rows wave, wave + W, ...; of every second one four groups' scales of
// 64 rows, if the wave is one of the first kEights / 8.
template <int kEights, int W>
struct SideLoads {
    static constexpr int kPer = kEights / W, kScaleWaves = kEights / 8;
    static_assert(kEights % W == 0, "every wave loads as much as the others");
    const uint8_t *codes, *scales;          // of the tile's first row
    uint32_t code_at[kPer], scale_at;       // this lane's rows from there

    __device__ __forceinline__ void start(const uint8_t *c, const uint8_t *s, int64_t row0, int64_t rows, int64_t blocks, int wave,
                                          int scale_wave, int lane)
    {
        codes = c + row0 * blocks * 16;
        scales = s + row0 * blocks;
        const int most = rows - row0 < kEights * 8 ? (int)(rows - row0) - 1 : kEights * 8 - 1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int place = (wave + W * i) * 8 + lane / 8;
            const uint32_t row = place < most ? place : most;       // past the end the last row again, stored nowhere
            code_at[i] = row * (uint32_t)blocks * 16 + block(lane, wave + W * i) * 16;
        }
        const int place = scale_wave * 64 + lane;
        scale_at = (uint32_t)(place < most ? place : most) * (uint32_t)blocks;
    }
    static __device__ __forceinline__ int block(int lane, int eight) { return (lane & 7) ^ ((eight * 8 + lane / 8) >> 1 & 7); }
    // eight i of this wave, from step `at` on, into the buffer at LDS address `to`; `one`: a row has no second step
    __device__ __forceinline__ void issue(int i, uint32_t to, int64_t at, bool one, int wave, int lane) const
    {
        const uint32_t second = one && block(lane, wave + W * i) >= 4 ? 64 : 0;
        direct_load(to + (wave + W * i) * 1024, codes + at * 64, code_at[i] - second);
    }
    __device__ __forceinline__ void issue_scales(uint32_t to, int64_t group) const { direct_load(to, scales + group * 4, scale_at); }
};

// 32 rows of a step in registers.
struct Rows32 {
    u32x4 codes[2];
    uint32_t scales;

    // rows 32 i .. 32 i + 31 of a side's pair, its first step or its second, and of its scales, `group` of the four there
    __device__ __forceinline__ void read(const uint8_t *side, const uint8_t *side_scales, int i, int second, int group, int lane)
    {
        const int r = lane & 31, h = lane >> 5;
        const uint8_t *const row = side + i * 4096 + r * 128;
        const int swizzle = (h ^ (r >> 1 & 7)) * 16;
        codes[0] = *reinterpret_cast<const u32x4 *>(row + (swizzle ^ second * 64));
        codes[1] = *reinterpret_cast<const u32x4 *>(row + (swizzle ^ (second * 64 + 32)));
        scales = *reinterpret_cast<const uint32_t *>(side_scales + (i * 32 + r) * 16 + group * 4);
    }
};

// f(0), f(1), ... with the numbers known when the program is built.
template <int... kNumbers, typename F>
__device__ __forceinline__ void each_phase(std::integer_sequence<int, kNumbers...>, F f)
{
    (f(std::integral_constant<int, kNumbers>{}), ...);
}

// A tile of results in LDS to memory, as far as `rows` and `cols` go.
template <int kThreadsOf, int kRows, int kElems, int kBytes>
__device__ __forceinline__ void store_tile(const uint8_t *tile, uint16_t *out, int64_t stride, int64_t rows, int64_t cols)
{
    constexpr int kLanes = kElems / 8;
    const int col = threadIdx.x % kLanes * 8;
#pragma unroll 4
    for (int row = threadIdx.x / kLanes; row < kRows; row += kThreadsOf / kLanes) {
        if (row < rows) store_row8(out + row * stride, col, cols, *reinterpret_cast<const u32x4 *>(tile + row * kBytes + col * 2));
    }
}

template <int WN, int WM, int FN, int FM, int kBuffers>
__global__ __launch_bounds__(64 * WN * WM) void product_tiles_kernel(Global<const uint8_t> xc, Global<const uint8_t> xs,
                                                                     Global<const uint8_t> wc, Global<const uint8_t> ws,
                                                                     Global<uint16_t> out, int32_t M, int32_t N, int32_t groups,
                                                                     int64_t out_stride, uint32_t tiles_n, uint32_t tiles_m)
{
    constexpr int W = WN * WM, kEightN = WN * FN * 4, kEightM = WM * FM * 4;
    constexpr int kSideN = kEightN * 1024, kPair = kSideN + kEightM * 1024;
    constexpr int kScalesN = kEightN * 128, kScales = kScalesN + kEightM * 128;
    constexpr int kWindows = kBuffers / 2 + 1;                      // fours of groups that the pairs in LDS are of
    static_assert(kBuffers % 2 == 0, "a pair's place among the four groups whose scales it shares is known from its buffer");
    __shared__ __align__(1024) uint8_t lds[kBuffers * kPair + kWindows * kScales];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5;
    const uint32_t tile_n = blockIdx.x % tiles_n, tile_m = blockIdx.x / tiles_n;
    const int64_t n0 = (int64_t)tile_n * (kEightN * 8), m0 = (int64_t)tile_m * (kEightM * 8);
    const int64_t blocks = (int64_t)groups * 4;
    using LoadsN = SideLoads<kEightN, W>;
    using LoadsM = SideLoads<kEightM, W>;
    // the waves share out the scales: one load of either side each, or one of one side
    constexpr int kScaleN = LoadsN::kScaleWaves, kScaleM = LoadsM::kScaleWaves;
    constexpr bool kBoth = kScaleN + kScaleM > W;
    static_assert(kScaleN <= W && kScaleM <= W, "at most one load of a side");
    LoadsN wl;
    LoadsM xl;
    const int scale_m = kBoth ? wave : wave - kScaleN;
    wl.start(wc, ws, n0, N, blocks, wave, wave, lane);
    xl.start(xc, xs, m0, M, blocks, wave, scale_m, lane);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // Scales come four groups at a time; the last four of a row may begin inside the four before.
    auto window = [&](int step) { return (step & ~3) + 4 <= groups ? step & ~3 : groups - 4; };
    // A part of the loads of the pair that begins at `step`; phase: step % (2 * kBuffers), known when the program is built.
    constexpr int kParts = 4 * FM;
    auto issue = [&](int step, auto phase, int part) {
        constexpr int kPhase = decltype(phase)::value;
        const uint32_t to = base + kPhase / 2 * kPair;
        if (kPhase % 4 == 0 && part == 0) {     // past the end, the last four again
            const uint32_t scales = base + kBuffers * kPair + (uint32_t)(step / 4 % kWindows) * kScales;
            const int from = window(step);
            if (kScaleN == W || wave < kScaleN) wl.issue_scales(scales + wave * 1024, from);
            if (kBoth && kScaleM == W) {
                xl.issue_scales(scales + kScalesN + scale_m * 1024, from);
            } else if (scale_m >= 0 && scale_m < kScaleM) {
                xl.issue_scales(scales + kScalesN + scale_m * 1024, from);
            }
        }
        const int64_t at = step < groups ? step : groups - 1;               // past the end: loaded again, not used
        const bool one = at + 1 == groups;
#pragma unroll
        for (int i = 0; i < LoadsN::kPer; ++i) {
            if (i * kParts / LoadsN::kPer == part) wl.issue(i, to, at, one, wave, lane);
        }
#pragma unroll
        for (int i = 0; i < LoadsM::kPer; ++i) {
            if (i * kParts / LoadsM::kPer == part) xl.issue(i, to + kSideN, at, one, wave, lane);
        }
    };
    v16f sum[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) sum[i][j] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};

    // Of w a lane holds this line of results' rows and the next line's, of x all of this step's and those of the next.
    Rows32 w[2], x[2][FM];
    static_assert(FN % 2 == 0 && FM <= FN, "a step asks for the next one's rows of x line by line");
    const int part_n = wave % WN, part_m = wave / WN;
    auto scales = [&](int step) { return lds + kBuffers * kPair + (uint32_t)(step / 4 % kWindows) * kScales; };
    auto read_w = [&](Rows32 &to, int step, int phase, int i) {
        to.read(lds + phase / 2 * kPair, scales(step), part_n * FN + i, phase % 2, (step - window(step)) & 3, lane);
    };
    auto read_x = [&](Rows32 &to, int step, int phase, int j) {
        to.read(lds + phase / 2 * kPair + kSideN, scales(step) + kScalesN, part_m * FM + j, phase % 2, (step - window(step)) & 3, lane);
    };
    using std::integral_constant;
    constexpr int kPhases = 2 * kBuffers, kPairLoads = LoadsN::kPer + LoadsM::kPer;     // of a wave, and its scales
    each_phase(std::make_integer_sequence<int, kBuffers - 1>{}, [&](auto pair) {
        constexpr int kPairOf = decltype(pair)::value;
#pragma unroll
        for (int part = 0; part < kParts; ++part) issue(2 * kPairOf, integral_constant<int, 2 * kPairOf>{}, part);
    });
#pragma unroll
    for (int part = 0; part < FM; ++part) issue(kPhases - 2, integral_constant<int, kPhases - 2>{}, part);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kBuffers - 2) * kPairLoads + kPairLoads / 4) : "memory");
#pragma unroll
    for (int j = 0; j < FM; ++j) read_x(x[0][j], 0, 0, j);
    read_w(w[0], 0, 0, 0);
    // What else a line has to do goes between its instructions, a little at a time: a wave issues in order.
    auto step = [&](int at, auto phase) {
        constexpr int kPhase = decltype(phase)::value, kNow = kPhase % 2, kNext = (kPhase + 1) % kPhases;
        constexpr bool kSecond = kPhase % 2 == 1;
        uint32_t sx[FM];
#pragma unroll
        for (int j = 0; j < FM; ++j) sx[j] = x[kNow][j].scales >> (8 * h);
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const uint32_t sw = w[i % 2].scales >> (8 * h);
            if (kSecond && i + 1 == FN) {
                // the next pair is in LDS for all waves, and this one has been read by all: its buffer is free
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kBuffers - 2) * kPairLoads) : "memory");
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                sum[i][j] = multiply<0>(w[i % 2].codes[0], sw, x[kNow][j].codes[0], sx[j], sum[i][j]);
                if (j == 0) {
                    if (i + 1 < FN) {
                        read_w(w[(i + 1) % 2], at, kPhase, i + 1);
                    } else {
                        read_w(w[0], at + 1, kNext, 0);
                    }
                }
                if (kSecond && i + 1 == FN) {
                    read_x(x[1 - kNow][j], at + 1, kNext, j);
                } else if (!kSecond && j == 1 % FM && i < FM) {
                    read_x(x[1 - kNow][i], at + 1, kNext, i);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                sum[i][j] = multiply<2>(w[i % 2].codes[1], sw, x[kNow][j].codes[1], sx[j], sum[i][j]);
                // (four loads in a row instead of one an instruction: 277 us for 8192 cubed, sixteen: 298)
                if (kSecond && i + 1 == FN) issue(at + kPhases - 1, integral_constant<int, kPhase - 1 + !kSecond>{}, j);
                if (!kSecond && i < 3) issue(at + kPhases - 2, integral_constant<int, (kPhase + kPhases - 2) % kPhases>{}, (i + 1) * FM + j);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!kSecond && i + 1 == FN) {
#pragma unroll
                for (int part = (FN + 1) * FM; part < kParts; ++part) issue(at + kPhases - 2, integral_constant<int, (kPhase + kPhases - 2) % kPhases>{}, part);
            }
        }
    };
    // No branch inside a round: a compiler that may moves the instructions of one step past the next one's wait.
    int at = 0;
    for (; at + kPhases <= groups; at += kPhases)
        each_phase(std::make_integer_sequence<int, kPhases>{}, [&](auto phase) { step(at + decltype(phase)::value, phase); });
    each_phase(std::make_integer_sequence<int, kPhases - 1>{}, [&](auto phase) {
        if (at + decltype(phase)::value < groups) step(at + decltype(phase)::value, phase);
    });
    // What was loaded past the end lands, all waves have read: LDS takes the results, bf16, a row of x after the other, from where
    // they leave in rows as long as the tile.  (Stored from registers, 32 bytes a row at a time, they took 2.5 us longer a tile,
    // and twice that where a row begins at an odd element.)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    constexpr int kRowElems = WN * FN * 32, kRowBytes = kRowElems * 2 + 16, kRows = WM * FM * 32;
    static_assert(kRows * kRowBytes <= kBuffers * kPair + kWindows * kScales, "the results take the codes' place");
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        uint8_t *const row = lds + ((part_m * FM + j) * 32 + (lane & 31)) * kRowBytes;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
#pragma unroll
            for (int q = 0; q < 4; q += 2) {        // a lane has four outputs from 8 q + 4 h on; after the exchange eight of one q
                const v16f &s = sum[i][j];
                auto lo = __builtin_amdgcn_permlane32_swap(narrow_bf16x2(s[4 * q], s[4 * q + 1]),
                                                           narrow_bf16x2(s[4 * q + 4], s[4 * q + 5]), false, false);
                auto hi = __builtin_amdgcn_permlane32_swap(narrow_bf16x2(s[4 * q + 2], s[4 * q + 3]),
                                                           narrow_bf16x2(s[4 * q + 6], s[4 * q + 7]), false, false);
                *reinterpret_cast<u32x4 *>(row + ((part_n * FN + i) * 32 + (q + h) * 8) * 2) = u32x4{lo[0], hi[0], lo[1], hi[1]};
            }
        }
    }
    __syncthreads();
    store_tile<64 * W, kRows, kRowElems, kRowBytes>(lds, out + m0 * out_stride + n0, out_stride, M - m0, N - n0);
}

}  // namespace mx4
}  // namespace equarx
