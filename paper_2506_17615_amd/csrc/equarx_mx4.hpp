// Device code of the 4-bit microscaled format: quantizing rows, reading them back, and the product of packed rows.
#pragma once

#include <type_traits>

#include "equarx_device.hpp"

namespace equarx {
namespace mx4 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 16 bytes at any even address: rows of any stride are read and written whole where they lie
typedef u32x4 u32x4_anywhere __attribute__((aligned(2)));

constexpr int kBlock = 32, kGroup = 128;

// n / d for n < 2^31 by a multiplication, d fixed for a launch (Granlund and Montgomery's round-up form).
struct Divisor {
    uint32_t magic, shift, d;
    explicit Divisor(uint32_t by) : magic(0), shift(0), d(by)
    {
        while (((uint64_t)1 << shift) < d) ++shift;
        magic = (uint32_t)((((((uint64_t)1 << shift) - d) << 32) / d) + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, magic) + n) >> shift; }
};

// ---------------------------------------------------------------- rows of bf16

// Elements [col, col + 8) of a row of `cols`; zeros past its end.
__device__ __forceinline__ u32x4 load_row8(const uint16_t *row, int64_t col, int64_t cols)
{
    if (col + 8 <= cols) return *reinterpret_cast<const u32x4_anywhere *>(row + col);
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = col + i < cols ? row[col + i] : 0;
    return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}

__device__ __forceinline__ void store_row8(uint16_t *row, int64_t col, int64_t cols, const u32x4 &v)
{
    if (col + 8 <= cols) {
        *reinterpret_cast<u32x4_anywhere *>(row + col) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (col + i < cols) row[col + i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
    }
}

// ---------------------------------------------------------------- one block's scale and codes

// The larger of each half of two words, as unsigned 16-bit numbers: magnitudes of bf16 numbers are ordered like their
// patterns.
__device__ __forceinline__ uint32_t umax16x2(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// The scale byte of a block whose largest magnitude has the bf16 pattern `top`.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const uint32_t e = top >> 7;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// 2^(byte - 127) as the instructions take it: they read the exponent field alone.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

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

// ---------------------------------------------------------------- rows <-> packed rows
// A lane has eight elements, a quad a block, a row of sixteen lanes a group: `units` pieces of eight in all, the
// padding among them, `unit` counting through the packed rows.

__global__ __launch_bounds__(256) void quantize_rows_kernel(Global<const uint16_t> x, int64_t x_stride, Global<uint8_t> codes,
                                                            Global<uint8_t> scales, int64_t cols, uint32_t units,
                                                            const Divisor row_units)
{
    const uint32_t unit = blockIdx.x * 256 + threadIdx.x;
    if (unit >= units) return;                                  // whole rows of sixteen lanes: units is a multiple of 16
    const uint32_t row = row_units.of(unit);
    const int64_t col = (int64_t)(unit - row * row_units.d) * 8;
    const u32x4 v = load_row8(x + row * x_stride, col, cols);
    uint32_t top = magnitudes_max(v);
    top = umax(top & 0xffff, top >> 16);
    top = umax(top, dpp_read<0xB1>(top));
    top = umax(top, dpp_read<0x4E>(top));
    const uint32_t byte = scale_byte(top);
    reinterpret_cast<uint32_t *>((uint8_t *)codes)[unit] = byte == 255 ? 0 : codes_of(v, scale_of(byte));
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
// One 16x16x128 matrix instruction takes 128 elements of 16 rows of w and of 16 rows of x: lane l has row l % 16 and
// its block l / 16 of four, with that block's scale.  Its result lane l has column l % 16 (a row of x) and the four rows
// of w 4 * (l / 16) + 0 .. 3: four consecutive outputs.

struct Packed {
    const uint8_t *codes, *scales;
    int64_t rows, blocks;
};

struct Fragment {
    u32x4 codes;
    uint32_t scale;
};

__device__ __forceinline__ Fragment load_fragment(const uint8_t *codes, const uint8_t *scales, int64_t block)
{
    Fragment f;
    f.codes = *reinterpret_cast<const u32x4 *>(codes + block * 16);
    f.scale = scales[block];
    return f;
}

__device__ __forceinline__ v4f multiply(const Fragment &w, const Fragment &x, const v4f &sum)
{
    const v8i a = {(int)w.codes[0], (int)w.codes[1], (int)w.codes[2], (int)w.codes[3], 0, 0, 0, 0};
    const v8i b = {(int)x.codes[0], (int)x.codes[1], (int)x.codes[2], (int)x.codes[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, sum, 4, 4, 0, (int)w.scale, 0, (int)x.scale);
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

// Sixteen rows of w by MT * 16 rows of x in a workgroup, the sum over k cut into W parts, one for a wave, that are added
// in order.
template <int W, int MT>
__global__ __launch_bounds__(64 * W) void product_rows_kernel(Global<const uint8_t> xc, Global<const uint8_t> xs,
                                                              Global<const uint8_t> wc, Global<const uint8_t> ws,
                                                              Global<uint16_t> out, int32_t M, int32_t N, int32_t groups,
                                                              int64_t out_stride)
{
    __shared__ v4f part[W][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
    const int64_t blocks = (int64_t)groups * 4;
    const int64_t wr = n0 + r < N ? n0 + r : N - 1;
    v4f sum[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) sum[t] = v4f{0, 0, 0, 0};
    const uint8_t *const wcr = wc + wr * blocks * 16, *const wsr = ws + wr * blocks;
    for (int s = wave; s < groups; s += W) {
        const Fragment w = load_fragment(wcr, wsr, 4 * s + g);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int64_t m = m0 + 16 * t + r, xr = m < M ? m : M - 1;
            sum[t] = multiply(w, load_fragment(xc + xr * blocks * 16, xs + xr * blocks, 4 * s + g), sum[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = sum[t];
    __syncthreads();
    for (int t = wave; t < MT; t += W) {
        v4f total = part[0][t][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) total += part[i][t][lane];
        const int64_t m = m0 + 16 * t + r;
        if (m < M) store_out4(out + m * out_stride, n0 + 4 * g, N, total);
    }
}

// ---- large products
// A workgroup of WN x WM waves has WN * FN * 32 rows of w by WM * FM * 32 rows of x, a wave FN x FM results of 32 x 32 in
// registers.  A step is the 128 elements of a group, two 32x32x64 instructions a result, whose lane l has row l % 32 and block l / 32
// of two.  Codes come to LDS with direct loads of two steps, a pair, into one of two buffers: a pair is asked for when
// the one before last has been read, two steps before its own turn.
//
// In LDS a row of a pair is 128 bytes, a line of memory, and rows follow each other as the lanes of a direct load do, eight
// lanes a row (rows spread over distant lanes, or half lines, are more requests: 8192 cubed 383 and 291 us).  The eight blocks of
// row r stand in the order of their number xor r / 2 % 8, so that one block of sixteen rows is in all banks once.  Scales: the
// four bytes of a row and step are a word; a lane shifts it by its block and the instruction picks byte 0 or 2.  Rows' scales lie
// far apart, a line each, so that they are loaded for four steps at once (a word a step: half of all requests).

// One direct load of 16 bytes a lane: LDS `to` + lane * 16 <- `from` + `offset`.
__device__ __forceinline__ void direct_load(uint32_t to, const uint8_t *from, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}

// The longest row of codes whose 256 a lane's 32-bit offset reaches.
constexpr int64_t kMostTileGroups = (int64_t)1 << 16;

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

template <int kHalf>
__device__ __forceinline__ v16f multiply32(const Rows32 &w, uint32_t w_scale, const Rows32 &x, uint32_t x_scale, const v16f &sum)
{
    const u32x4 p = w.codes[kHalf], q = x.codes[kHalf];
    const v8i a = {(int)p[0], (int)p[1], (int)p[2], (int)p[3], 0, 0, 0, 0};
    const v8i b = {(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, sum, 4, 4, 2 * kHalf, (int)w_scale, 2 * kHalf, (int)x_scale);
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

template <int WN, int WM, int FN, int FM>
__global__ __launch_bounds__(64 * WN * WM) void product_tiles_kernel(Global<const uint8_t> xc, Global<const uint8_t> xs,
                                                                     Global<const uint8_t> wc, Global<const uint8_t> ws,
                                                                     Global<uint16_t> out, int32_t M, int32_t N, int32_t groups,
                                                                     int64_t out_stride, uint32_t tiles_n, uint32_t tiles_m)
{
    constexpr int W = WN * WM, kEightN = WN * FN * 4, kEightM = WM * FM * 4;
    constexpr int kSideN = kEightN * 1024, kPair = kSideN + kEightM * 1024;
    constexpr int kScalesN = kEightN * 128, kScales = kScalesN + kEightM * 128;
    __shared__ __align__(1024) uint8_t lds[2 * (kPair + kScales)];
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
    // A part of the loads of the pair that begins at `step`; phase: step % 4, known when the program is built.
    constexpr int kParts = 4 * FM;
    auto issue = [&](int step, auto phase, int part) {
        constexpr int kPhase = decltype(phase)::value;
        const uint32_t to = base + kPhase / 2 * kPair;
        if (kPhase == 0 && part == 0) {         // past the end, the last four again
            const uint32_t scales = base + 2 * kPair + (uint32_t)(step / 4 % 2) * kScales;
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
    auto scales = [&](int step) { return lds + 2 * kPair + (uint32_t)(step / 4 % 2) * kScales; };
    auto read_w = [&](Rows32 &to, int step, int phase, int i) {
        to.read(lds + phase / 2 * kPair, scales(step), part_n * FN + i, phase % 2, (step - window(step)) & 3, lane);
    };
    auto read_x = [&](Rows32 &to, int step, int phase, int j) {
        to.read(lds + phase / 2 * kPair + kSideN, scales(step) + kScalesN, part_m * FM + j, phase % 2, (step - window(step)) & 3, lane);
    };
    using std::integral_constant;
#pragma unroll
    for (int part = 0; part < kParts; ++part) issue(0, integral_constant<int, 0>{}, part);
#pragma unroll
    for (int part = 0; part < FM; ++part) issue(2, integral_constant<int, 2>{}, part);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((LoadsN::kPer + LoadsM::kPer) / 4) : "memory");
#pragma unroll
    for (int j = 0; j < FM; ++j) read_x(x[0][j], 0, 0, j);
    read_w(w[0], 0, 0, 0);
    // What else a line has to do goes between its instructions, a little at a time: a wave issues in order.
    auto step = [&](int at, auto phase) {
        constexpr int kPhase = decltype(phase)::value, kNow = kPhase % 2, kNext = (kPhase + 1) % 4;
        constexpr bool kSecond = kPhase % 2 == 1;
        uint32_t sx[FM];
#pragma unroll
        for (int j = 0; j < FM; ++j) sx[j] = x[kNow][j].scales >> (8 * h);
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const uint32_t sw = w[i % 2].scales >> (8 * h);
            if (kSecond && i + 1 == FN) {
                // the next pair is in LDS for all waves, and this one has been read by all: its buffer is free
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                sum[i][j] = multiply32<0>(w[i % 2], sw, x[kNow][j], sx[j], sum[i][j]);
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
                sum[i][j] = multiply32<1>(w[i % 2], sw, x[kNow][j], sx[j], sum[i][j]);
                // (four loads in a row instead of one an instruction: 277 us for 8192 cubed, sixteen: 298)
                if (kSecond && i + 1 == FN) issue(at + 3, integral_constant<int, (kPhase + 3) % 4>{}, j);
                if (!kSecond && i < 3) issue(at + 2, integral_constant<int, (kPhase + 2) % 4>{}, (i + 1) * FM + j);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!kSecond && i + 1 == FN) {
#pragma unroll
                for (int part = (FN + 1) * FM; part < kParts; ++part) issue(at + 2, integral_constant<int, (kPhase + 2) % 4>{}, part);
            }
        }
    };
    // No branch inside four steps: a compiler that may moves the instructions of one past the next one's wait.
    int at = 0;
    for (; at + 4 <= groups; at += 4) {
        step(at, integral_constant<int, 0>{});
        step(at + 1, integral_constant<int, 1>{});
        step(at + 2, integral_constant<int, 2>{});
        step(at + 3, integral_constant<int, 3>{});
    }
    if (at < groups) step(at, integral_constant<int, 0>{});
    if (at + 1 < groups) step(at + 1, integral_constant<int, 1>{});
    if (at + 2 < groups) step(at + 2, integral_constant<int, 2>{});
    // What was loaded past the end lands, all waves have read: LDS takes the results, bf16, a row of x after the other, from where
    // they leave in rows as long as the tile.  (Stored from registers, 32 bytes a row at a time, they took 2.5 us longer a tile,
    // and twice that where a row begins at an odd element.)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    constexpr int kRowElems = WN * FN * 32, kRowBytes = kRowElems * 2 + 16, kRows = WM * FM * 32;
    static_assert(kRows * kRowBytes <= (int)sizeof(lds), "the results take the codes' place");
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
