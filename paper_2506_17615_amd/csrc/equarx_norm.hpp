// Device code of the root-mean-square norm: of rows, and of rows that are the quantized reduction of P partial sums.
#pragma once

#include "equarx_rows.hpp"

namespace equarx {
namespace norm {

// What a row becomes: any of bf16, int8 with scales, packed 4 bits.
struct Outputs {
    Global<uint16_t> out;
    int64_t out_stride;
    Global<int8_t> codes;
    Global<float> scales;
    Global<uint8_t> mx_codes, mx_scales;
    int32_t block;          // of the int8 form
};

// What becomes a row: the residual stream (or null), g and eps.
struct Inputs {
    Global<uint16_t> residual;
    int64_t residual_stride;
    Global<const uint16_t> weight;
    double eps;
    int32_t one_plus;
};

// Where a thread works: `L` lanes have a row, L a multiple of 16; a row's lane l has the units of eight elements l, l + L, ...
template <int L>
struct Place {
    static constexpr int T = L < 256 ? 256 : L, kRows = T / L;
    int64_t row;
    int lane;
    bool any;
    __device__ __forceinline__ Place(int64_t rows)
    {
        const int in = L < 64 ? threadIdx.x / L : __builtin_amdgcn_readfirstlane(threadIdx.x / L);     // a wave's row is a scalar
        row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? in : 0);
        lane = threadIdx.x % L;
        any = kRows == 1 || row < rows;
    }
};

// ---------------------------------------------------------------- units of a row
// Where a wave has one row and all rows begin on sixteen bytes and end with a unit (kWhole), through a descriptor that ends with the row:
// nothing is behind a condition, so that all loads of a thread are asked for together (behind one each the compiler waited for the first
// two before it asked for the third: 4096 x 5376 to int8 42.5 us, 38.5 this way), and what is past the row's end is not read, zero, and not written.

template <int L, bool kWhole>
constexpr bool by_descriptor = kWhole && L >= 64;

template <int L, int K, bool kWhole, int kPolicy = 0>
__device__ __forceinline__ void load_units(const uint16_t *p, const Place<L> &at, int32_t cols, u32x4 (&v)[K])
{
    if constexpr (by_descriptor<L, kWhole>) {
        const auto row = bounded(p, at.any ? cols * 2 : 0);
#pragma unroll
        for (int k = 0; k < K; ++k)
            v[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(row, (at.lane + k * L) * 16, 0, kPolicy));
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t col = (at.lane + k * L) * 8;
            v[k] = u32x4{0, 0, 0, 0};
            if (at.any && col < cols) v[k] = kWhole || cols < 8 ? load_row8(p, col, cols) : load_row8_back(p, col, cols);
        }
    }
}

template <int L, bool kWhole, int kPolicy = 0>
__device__ __forceinline__ void store_unit(uint16_t *p, const Place<L> &at, int k, int32_t cols, const u32x4 &v)
{
    if constexpr (by_descriptor<L, kWhole>) {
        __builtin_amdgcn_raw_buffer_store_b128(v, bounded(p, at.any ? cols * 2 : 0), (at.lane + k * L) * 16, 0, kPolicy);
    } else {
        const int32_t col = (at.lane + k * L) * 8;
        if (at.any && col < cols) store_row8(p, col, cols, v);
    }
}

// ---------------------------------------------------------------- a row's sum

template <int kCtrl>
__device__ __forceinline__ double dpp_read64(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)dpp_read<kCtrl>((uint32_t)(b >> 32)) << 32 | dpp_read<kCtrl>((uint32_t)b));
}

__device__ __forceinline__ double join64(uint32_t low, uint32_t high)
{
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

// The sum over the L lanes of a row, in all of them; every lane of the workgroup calls it.
template <int L>
__device__ __forceinline__ double row_sum(double s)
{
    s += dpp_read64<0xB1>(s);
    s += dpp_read64<0x4E>(s);
    s += dpp_read64<0x141>(s);
    s += dpp_read64<0x140>(s);
    if (L == 16) return s;
    uint64_t b = __builtin_bit_cast(uint64_t, s);
    auto low = __builtin_amdgcn_permlane16_swap((uint32_t)b, (uint32_t)b, false, false);
    auto high = __builtin_amdgcn_permlane16_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    s = join64(low[0], high[0]) + join64(low[1], high[1]);
    b = __builtin_bit_cast(uint64_t, s);
    low = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false);
    high = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    s = join64(low[0], high[0]) + join64(low[1], high[1]);
    if (L > 64) {
        __shared__ double parts[L < 64 ? 1 : L / 64];
        if ((threadIdx.x & 63) == 0) parts[threadIdx.x / 64] = s;
        __syncthreads();
        s = parts[0];
#pragma unroll
        for (int i = 1; i < L / 64; ++i) s += parts[i];
    }
    return s;
}

// ---------------------------------------------------------------- what a row becomes

// The largest of the B / 8 lanes of a block, B known at the launch only: the steps of group_max_bits as far as they go.
__device__ __forceinline__ uint32_t block_max_bits(uint32_t m, int32_t block)
{
    m = umax(m, dpp_read<0xB1>(m));
    m = umax(m, dpp_read<0x4E>(m));
    if (block >= 64) m = umax(m, dpp_read<0x141>(m));
    if (block >= 128) m = umax(m, dpp_read<0x140>(m));
    if (block >= 256) {
        auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = umax(r[0], r[1]);
    }
    if (block >= 512) {
        auto r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        m = umax(r[0], r[1]);
    }
    return m;
}

__device__ __forceinline__ uint32_t top_of(const float (&y)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = umax(top, __float_as_uint(y[i]) & 0x7fffffffu);
    return top;
}

constexpr uint32_t kInfinity = 0x7f800000u;

// Q_B of a lane's eight values; a block that is not finite gets a NaN for its scale and zeros for its codes.
__device__ __forceinline__ u32x2 int8_of(const float (&y)[8], uint32_t top, int32_t block, float &scale)
{
    const uint32_t a = block_max_bits(top, block);
    float inv;
    block_quotients(__uint_as_float(a), scale, inv);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(y[i] * inv + kRoundMagic);
    u32x2 w = {gather_low_bytes(b[0], b[1], b[2], b[3]), gather_low_bytes(b[4], b[5], b[6], b[7])};
    if (a >= kInfinity) {
        scale = __uint_as_float(0x7fc00000u);
        w = u32x2{0, 0};
    }
    return w;
}

// A lane's eight values in 4 bits, the quad's block of 32 sharing the scale byte.
__device__ __forceinline__ uint32_t mx4_of(const float (&y)[8], uint32_t top, uint32_t &byte)
{
    top = umax(top, dpp_read<0xB1>(top));
    top = umax(top, dpp_read<0x4E>(top));
    byte = mx4::scale_byte(top >> 16);
    const float scale = mx4::scale_of(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
    return byte == 255 ? 0 : w;
}

// A thread's K units of a row, `h` what was added up in fp32 (h itself where there is no residual stream): the stream, the norm
// and its outputs.
//
//   h = bf16(..) -> residual;   i = fl32(1 / sqrt(sum_64(h^2) / cols + eps));   y = fl32(fl32(h i) g)
// The sum is taken in 64 bits, where its order does not reach i's last bit (but for one row in 10^8): the codes of the
// quantized forms, each of which one bit of i can tip over, depend on the row alone, not on how it was cut.  bf16, int8 and 4 bits
// are each rounded from y itself, once.
template <int L, int K, bool kWhole, bool kStreams>
__device__ __forceinline__ void finish_row(const Place<L> &at, u32x4 (&h)[K], const u32x4 (&r)[K], const u32x4 (&w)[K], int64_t cols,
                                           const Inputs &in, const Outputs &to)
{
    double sum = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[8];
        widen_bf16x8(h[k], f);
        if (in.residual.address) {
            float g[8];
            widen_bf16x8(r[k], g);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[k][i] = narrow_bf16x2(f[2 * i] + g[2 * i], f[2 * i + 1] + g[2 * i + 1]);
            store_unit<L, kWhole>(in.residual + at.row * in.residual_stride, at, k, (int32_t)cols, h[k]);
            widen_bf16x8(h[k], f);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double d = f[i];
            sum = __builtin_fma(d, d, sum);
        }
    }
    sum = row_sum<L>(sum);
    const int shift = 31 - __builtin_clz((uint32_t)to.block | 1u);       // a block is a power of two
    const float inverse = (float)(1.0 / __builtin_sqrt(sum / (double)cols + in.eps));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t unit = at.lane + k * L, col = unit * 8;
        float y[8], g[8];
        widen_bf16x8(h[k], y);
        widen_bf16x8(w[k], g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (in.one_plus) g[i] += 1.0f;
            y[i] = y[i] * inverse;
            if (in.weight.address) y[i] = y[i] * g[i];
            if (kWhole ? col >= cols : col + i >= cols) y[i] = 0.0f;        // 0 * infinity is not the row's
        }
        const bool real = at.any && col < cols;
        if (to.out.address) {
            const u32x4 v = {narrow_bf16x2(y[0], y[1]), narrow_bf16x2(y[2], y[3]), narrow_bf16x2(y[4], y[5]), narrow_bf16x2(y[6], y[7])};
            store_unit<L, kWhole, kStreams ? kNonTemporal : 0>(to.out + at.row * to.out_stride, at, k, (int32_t)cols, v);
        }
        const uint32_t top = top_of(y);
        if (to.codes.address) {                                     // whole blocks a row: whole units
            float scale;
            const u32x2 codes = int8_of(y, top, to.block, scale);
            if (real) {
                *reinterpret_cast<u32x2 *>((int8_t *)to.codes + at.row * cols + col) = codes;
                if ((col & (to.block - 1)) == 0) to.scales[at.row * (cols >> shift) + (col >> shift)] = scale;
            }
        }
        if (to.mx_codes.address) {                                  // rows are padded to whole sixteens of units
            uint32_t byte;
            const uint32_t codes = mx4_of(y, top, byte);
            uint32_t four = byte << (8 * ((threadIdx.x >> 2) & 3));
            four |= dpp_read<0x141>(four);
            four |= dpp_read<0x140>(four);
            const int64_t groups = (cols + mx4::kGroup - 1) / mx4::kGroup;
            if (at.any && unit < groups * 16) {
                reinterpret_cast<uint32_t *>((uint8_t *)to.mx_codes)[at.row * groups * 16 + unit] = codes;
                if ((threadIdx.x & 15) == 0) reinterpret_cast<uint32_t *>((uint8_t *)to.mx_scales)[at.row * groups + unit / 16] = four;
            }
        }
    }
}

// ---------------------------------------------------------------- rows of a tensor

// kStreams: a bf16 output that is written past the caches.
template <int L, int K, bool kWhole, bool kStreams>
__global__ __launch_bounds__(Place<L>::T) void rows_kernel(Global<const uint16_t> x, int64_t x_stride, int64_t rows, int64_t cols,
                                                           const Inputs in, const Outputs to)
{
    const Place<L> at(rows);
    u32x4 h[K], r[K], w[K];
    load_units<L, K, kWhole>(x + at.row * x_stride, at, (int32_t)cols, h);
    if (in.residual.address) load_units<L, K, kWhole>(in.residual + at.row * in.residual_stride, at, (int32_t)cols, r);
    if (in.weight.address) load_units<L, K, kWhole>(in.weight, at, (int32_t)cols, w);
    loads_first();
    finish_row<L, K, kWhole, kStreams>(at, h, r, w, cols, in, to);
}

// ---------------------------------------------------------------- rows that a reduction leaves
// The chain of chain_kernel over a row's blocks, B / 8 lanes each, whole blocks a row; its last dequantization is rounded to
// bf16, as equarx_reduce_fused writes it, and is the row that is normed.

// A: partials that are asked for together.  One at a time where rows are many (hence past the caches), short, or of any stride.  kWhole: of residual and output; the
// partials and the weight always are.
template <int B, int L, int K, int A, bool kWhole, bool kStreams>
__global__ __launch_bounds__(Place<L>::T) void reduced_kernel(int P, int64_t rows, int64_t cols, const Inputs in, const Outputs to,
                                                              const PartialTable tab)
{
    constexpr int G = B / kLaneElems;
    const Place<L> at(rows);
    u32x4 x[A][K], r[K] = {}, w[K] = {};
    float t[K][8] = {};
    // a wave behind the row's end has nothing to add up
    const int wave_lane = __builtin_amdgcn_readfirstlane(at.lane & ~63);
    const int batches = L > 64 && (int64_t)wave_lane * 8 >= cols ? 0 : P;
    for (int j = 0; j < batches; j += A) {
#pragma unroll
        for (int a = 0; a < A; ++a) load_units<L, K, true, A == 1 ? kNonTemporal : 0>(tab.x[j + a] + at.row * cols, at, (int32_t)cols, x[a]);
        if (j == 0) {
            if (in.residual.address) load_units<L, K, kWhole>(in.residual + at.row * in.residual_stride, at, (int32_t)cols, r);
            if (in.weight.address) load_units<L, K, true>(in.weight, at, (int32_t)cols, w);
        }
        if (A > 1) loads_first();
#pragma unroll
        for (int a = 0; a < A; ++a) {
            if (A > 1 && j + a >= P) break;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float f[8];
                widen_bf16x8(x[a][k], f);
                if (j + a == 0) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[k][i] = f[i];
                    continue;
                }
                float c[8], s;
                quantize_lane_f<G>(t[k], c, s);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[k][i] = __builtin_fmaf(c[i], s, f[i]);
            }
        }
    }
    u32x4 h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float c[8], s;
        quantize_lane_f<G, true>(t[k], c, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[k][i] = narrow_bf16x2(c[2 * i] * s, c[2 * i + 1] * s);
    }
    finish_row<L, K, kWhole, kStreams>(at, h, r, w, cols, in, to);
}

}  // namespace norm
}  // namespace equarx
