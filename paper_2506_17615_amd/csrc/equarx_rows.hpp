// Rows of bf16 at any stride, eight elements a lane, and the packed 4-bit format's scale: what the kernels over rows share.
#pragma once

#include "equarx_device.hpp"

namespace equarx {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 16 bytes at any even address: rows of any stride are read and written whole where they lie
typedef u32x4 u32x4_anywhere __attribute__((aligned(2)));

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

// The other lane's value, zero where the row of sixteen has none.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ uint32_t shifted(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, 0xf, false);
}

// A lane's value and those before it, as `add` adds; add(v, 0) is v.
template <typename F>
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, F add)
{
    v = add(v, shifted<0x111>(v));              // row_shr:1, 2, 4, 8
    v = add(v, shifted<0x112>(v));
    v = add(v, shifted<0x114>(v));
    v = add(v, shifted<0x118>(v));
    v = add(v, shifted<0x142, 0xa>(v));         // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    return add(v, shifted<0x143, 0xc>(v));
}

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

// Eight elements without the first `by`, zeros after them.
__device__ __forceinline__ u32x4 drop_elements(const u32x4 &v, int32_t by)
{
    const uint64_t low = (uint64_t)v.y << 32 | v.x, high = (uint64_t)v.w << 32 | v.z;
    const int bits = (by & 3) * 16;
    uint64_t l = low >> bits | (high << 1) << (63 - bits), h = high >> bits;
    if (by >= 4) {
        l = h;
        h = 0;
    }
    if (by >= 8) l = 0;
    return u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// load_row8 without a branch, for rows of eight elements and more: what would reach past the end is read from its last eight.
__device__ __forceinline__ u32x4 load_row8_back(const uint16_t *row, int32_t col, int32_t cols)
{
    const int32_t from = col + 8 <= cols ? col : cols - 8;
    const u32x4 v = *reinterpret_cast<const u32x4_anywhere *>(row + from);
    return drop_elements(v, col - from);
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

namespace mx4 {

constexpr int kBlock = 32, kGroup = 128;

// The scale byte of a block whose largest magnitude has the bf16 pattern `top`.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const uint32_t e = top >> 7;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// 2^(byte - 127) as the instructions take it: they read the exponent field alone.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace mx4
}  // namespace equarx
