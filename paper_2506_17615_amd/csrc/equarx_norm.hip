// Host side of the norms: argument validation, kernel selection and launch.
#include "equarx.h"

#include <cmath>

#include "equarx_launch.hpp"
#include "equarx_norm.hpp"

namespace {

using namespace equarx;
using namespace equarx::host;
using namespace equarx::norm;

constexpr int64_t kMostRows = INT32_MAX, kMostCols = EQUARX_NORM_MAX_COLS;
constexpr int kInPlace = 1;

int check_rows(int64_t rows, int64_t cols, int64_t stride)
{
    return stride < cols || stride > ((int64_t)1 << 40) / rows ? EQUARX_BAD_SHAPE : EQUARX_OK;
}

inline size_t row_bytes(int64_t rows, int64_t cols, int64_t stride) { return (size_t)((rows - 1) * stride + cols) * 2; }

// Everything but what is normed; rows and cols at least 1.  kInPlace: the input that `out` may be.
int check_norm(void *residual, int64_t residual_stride, const void *weight, int64_t rows, int64_t cols, double eps, uint32_t flags,
               const equarx_norm_outputs *to, Aliasing &mem)
{
    if (!(eps >= 0) || !std::isfinite(eps) || (flags & ~EQUARX_NORM_ONE_PLUS) || ((flags & EQUARX_NORM_ONE_PLUS) && !weight))
        return EQUARX_BAD_SHAPE;
    if (!to) return EQUARX_NULL_POINTER;
    if (!to->codes != !to->scales || !to->mx4_codes != !to->mx4_scales) return EQUARX_NULL_POINTER;
    if (!to->out_bf16 && !to->codes && !to->mx4_codes) return EQUARX_NULL_POINTER;
    if (to->codes && !block_ok(to->block)) return EQUARX_BAD_BLOCK;
    if (to->codes && cols % to->block != 0) return EQUARX_BAD_SHAPE;
    if (to->out_bf16) {
        if (int st = check_rows(rows, cols, to->out_stride)) return st;
    }
    if (residual) {
        if (int st = check_rows(rows, cols, residual_stride)) return st;
    }
    const void *const all[] = {residual, weight, to->out_bf16, to->codes, to->scales, to->mx4_codes, to->mx4_scales};
    for (const void *p : all) {
        if (misaligned(p, kAlign)) return EQUARX_MISALIGNED;
    }
    mem.reads(weight, (size_t)cols * 2);
    mem.writes(residual, row_bytes(rows, cols, residual_stride));
    if (to->out_bf16) mem.writes(to->out_bf16, row_bytes(rows, cols, to->out_stride), kInPlace);
    if (to->codes) {
        mem.writes(to->codes, (size_t)(rows * cols));
        mem.writes(to->scales, (size_t)(rows * cols) / to->block * sizeof(float));
    }
    const size_t groups = (size_t)((cols + mx4::kGroup - 1) / mx4::kGroup);
    mem.writes(to->mx4_codes, (size_t)rows * groups * (mx4::kGroup / 2));
    mem.writes(to->mx4_scales, (size_t)rows * groups * (mx4::kGroup / mx4::kBlock));
    return mem.check();
}

Inputs inputs_of(void *residual, int64_t residual_stride, const void *weight, double eps, uint32_t flags)
{
    return {static_cast<uint16_t *>(residual), residual_stride, static_cast<const uint16_t *>(weight), eps,
            (flags & EQUARX_NORM_ONE_PLUS) != 0};
}

Outputs outputs_of(const equarx_norm_outputs &to)
{
    return {static_cast<uint16_t *>(to.out_bf16), to.out_stride, to.codes, to.scales, to.mx4_codes, to.mx4_scales, to.block};
}

// Do all rows of the residual stream and of the output begin on sixteen bytes?
bool in_units(const Inputs &in, const Outputs &to)
{
    return (!in.residual.address || in.residual_stride % 8 == 0) && (!to.out.address || to.out_stride % 8 == 0);
}

// The same from row `at` on.
void advance(Inputs &in, Outputs &to, int64_t at, int64_t cols)
{
    const int64_t groups = (cols + mx4::kGroup - 1) / mx4::kGroup;
    if (in.residual.address) in.residual.address += (uint64_t)(at * in.residual_stride) * 2;
    if (to.out.address) to.out.address += (uint64_t)(at * to.out_stride) * 2;
    if (to.codes.address) {
        to.codes.address += (uint64_t)(at * cols);
        to.scales.address += (uint64_t)(at * cols / to.block) * sizeof(float);
    }
    if (to.mx_codes.address) {
        to.mx_codes.address += (uint64_t)(at * groups) * (mx4::kGroup / 2);
        to.mx_scales.address += (uint64_t)(at * groups) * (mx4::kGroup / mx4::kBlock);
    }
}

// From so many elements on bf16 outputs are written past the caches, which would not hold them for the next call as they would a decode
// step's.  Measured on MI355X, us with ordinary stores -> past the caches: 4096 x 5376 32.1 -> 29.2, 16384 x 1024 23.1 -> 20.4, 1024 x 5376
// 9.6 -> 9.1.  Rows that are not read through a descriptor have ordinary stores.
constexpr int64_t kStreamFrom = (int64_t)4 << 20;

template <int L_, int K_, int A_ = 1>
struct Cut {
    static constexpr int L = L_, K = K_, A = A_;
};

// f(cut) with the lanes that have a row, and their units: the fewest lanes, four waves at most while they hold a row in registers, since what counts is
// how many rows are on their way.
template <typename F>
void with_cut(int64_t cols, F f)
{
    if (cols <= 16 * 8) {
        f(Cut<16, 1>{});
    } else if (cols <= 64 * 8) {
        f(Cut<64, 1>{});
    } else if (cols <= 64 * 16) {
        f(Cut<64, 2>{});
    } else if (cols <= 256 * 8) {
        f(Cut<256, 1>{});
    } else if (cols <= 256 * 16) {
        f(Cut<256, 2>{});
    } else if (cols <= 256 * 24) {
        f(Cut<256, 3>{});
    } else if (cols <= 256 * 32) {
        f(Cut<256, 4>{});
    } else if (cols <= 1024 * 16) {
        f(Cut<1024, 2>{});
    } else {
        f(Cut<1024, 4>{});
    }
}


// Few rows of partial sums: sixteen waves a row, and up to sixteen partial sums asked for at once; what is left is the arithmetic of the chain
// on as many CUs as there are rows, 0.4 us a partial sum of 64 x 5376.  Many: as other rows, the partial sums one after the other, past the
// caches (8 of 4096 x 5376: 96.6 us with ordinary loads, 81.4 without, 79 with the output's stores past them too: 6.1 TB/s).  Measured on MI355X, us one
// way and the other, 5376 columns:
//     rows      P = 4            8               16
//     128     7.5    5.4          --         19.1   11.2
//     256     8.6    6.8     12.4    9.4     20.1   14.2
//     512    11.4   10.9     13.3   14.7     19.8   23.2
//     1024   17.9   16.8     22.9   28.6     36.7     --
// Other widths go by the same rule and were not measured.  Rows of up to 1024 columns, and all whose residual or output does not begin on sixteen
// bytes, ask for one partial sum after the other however few they are; above 16384 columns a lane keeps 68 bytes of its four units in scratch.
template <typename F>
void with_reduced_cut(int64_t rows, int64_t cols, int P, F f)
{
    if (rows > (P <= 4 ? 1024 : 256) || cols <= 64 * 16) {
        with_cut(cols, f);
    } else if (cols > 1024 * 16) {
        f(Cut<1024, 4, 4>{});
    } else if (cols > 1024 * 8) {
        f(Cut<1024, 2, 8>{});
    } else if (P <= 4) {
        f(Cut<1024, 1, 4>{});
    } else if (P <= 8) {
        f(Cut<1024, 1, 8>{});
    } else {
        f(Cut<1024, 1, 16>{});
    }
}

// Up to a row for every CU a row has a workgroup of sixteen waves, a unit a lane: 256 x 8192 5.3 -> 4.8 us, 1 x 8192 4.7 -> 4.4; 512 rows gain nothing,
// 1024 x 5376 loses (10.2 -> 10.7).
template <typename F>
void with_rows_cut(int64_t rows, int64_t cols, F f)
{
    if (rows <= 256 && cols > 256 * 8 && cols <= 1024 * 8) {
        f(Cut<1024, 1>{});
    } else {
        with_cut(cols, f);
    }
}

// f(first row, rows) for launches of at most 2^20 workgroups.
template <int L, typename F>
void in_row_pieces(int64_t rows, F f)
{
    constexpr int64_t kMost = (int64_t)Place<L>::kRows << 20;
    for (int64_t at = 0; at < rows; at += kMost) f(at, rows - at < kMost ? rows - at : kMost);
}

template <int L>
unsigned workgroups(int64_t rows)
{
    return (unsigned)((rows + Place<L>::kRows - 1) / Place<L>::kRows);
}

template <int B>
void launch_reduced(const PartialTable &partials, int P, int64_t rows, int64_t cols, const Inputs &in, const Outputs &to, LaunchCtx &ctx)
{
    auto launch = [&](auto cut, auto kernel) {
        constexpr int L = decltype(cut)::L;
        in_row_pieces<L>(rows, [&](int64_t at, int64_t count) {
            Inputs i = in;
            Outputs o = to;
            advance(i, o, at, cols);
            PartialTable tab = partials;
            for (int j = 0; j < kMaxPartials; ++j) tab.x[j] += at * cols;
            ctx.launch(kernel, workgroups<L>(count), Place<L>::T, P, count, cols, i, o, tab);
        });
    };
    if (!in_units(in, to)) {                                    // seldom: three cuts are enough
        if (cols <= 64 * 16) {
            launch(Cut<64, 2>{}, reduced_kernel<B, 64, 2, 1, false, false>);
        } else if (cols <= 256 * 32) {
            launch(Cut<256, 4>{}, reduced_kernel<B, 256, 4, 1, false, false>);
        } else {
            launch(Cut<1024, 4>{}, reduced_kernel<B, 1024, 4, 1, false, false>);
        }
        return;
    }
    with_reduced_cut(rows, cols, P, [&](auto cut) {
        constexpr int L = decltype(cut)::L, K = decltype(cut)::K, A = decltype(cut)::A;
        if constexpr (L * 8 >= B) {                             // as cols >= B
            constexpr bool kMayStream = A == 1 && L > 64;
            launch(cut, rows * cols >= kStreamFrom ? reduced_kernel<B, L, K, A, true, kMayStream> : reduced_kernel<B, L, K, A, true, false>);
        }
    });
}

}  // namespace

extern "C" {

int equarx_norm(const void *x_bf16, int64_t x_stride, void *residual_bf16, int64_t residual_stride, const void *weight_bf16,
                int64_t rows, int64_t cols, double eps, uint32_t flags, const equarx_norm_outputs *outputs, void *stream)
{
    LaunchCtx ctx(stream);
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostCols) return EQUARX_BAD_SHAPE;
    if (rows == 0 || cols == 0) return EQUARX_OK;
    if (int st = check_rows(rows, cols, x_stride)) return st;
    if (!x_bf16) return EQUARX_NULL_POINTER;
    if (misaligned(x_bf16, kAlign)) return EQUARX_MISALIGNED;
    Aliasing mem;
    mem.reads(x_bf16, row_bytes(rows, cols, x_stride), kInPlace);
    if (int st = check_norm(residual_bf16, residual_stride, weight_bf16, rows, cols, eps, flags, outputs, mem)) return st;
    const Inputs in = inputs_of(residual_bf16, residual_stride, weight_bf16, eps, flags);
    const Outputs to = outputs_of(*outputs);
    const bool whole = cols % 8 == 0 && x_stride % 8 == 0 && in_units(in, to);
    with_rows_cut(rows, cols, [&](auto cut) {
        constexpr int L = decltype(cut)::L, K = decltype(cut)::K;
        in_row_pieces<L>(rows, [&](int64_t at, int64_t count) {
            Inputs i = in;
            Outputs o = to;
            advance(i, o, at, cols);
            constexpr bool kMayStream = by_descriptor<L, true>;
            ctx.launch(!whole ? rows_kernel<L, K, false, false> : rows * cols < kStreamFrom ? rows_kernel<L, K, true, false> : rows_kernel<L, K, true, kMayStream>,
                       workgroups<L>(count), Place<L>::T,
                       static_cast<const uint16_t *>(x_bf16) + at * x_stride, x_stride, count, cols, i, o);
        });
    });
    return ctx.status();
}

int equarx_norm_reduced(const void *const *partials_bf16, int32_t P, int32_t block, void *residual_bf16, int64_t residual_stride,
                        const void *weight_bf16, int64_t rows, int64_t cols, double eps, uint32_t flags,
                        const equarx_norm_outputs *outputs, void *stream)
{
    LaunchCtx ctx(stream);
    if (!block_ok(block)) return EQUARX_BAD_BLOCK;
    if (P < 1 || P > EQUARX_MAX_PARTIALS || rows < 0 || cols < 0 || rows > kMostRows || cols > kMostCols || cols % block != 0)
        return EQUARX_BAD_SHAPE;
    if (rows == 0 || cols == 0) return EQUARX_OK;
    if (int st = check_rows(rows, cols, cols)) return st;
    if (!partials_bf16) return EQUARX_NULL_POINTER;
    Aliasing mem;
    PartialTable tab;
    for (int32_t i = 0; i < P; ++i) {
        if (!partials_bf16[i]) return EQUARX_NULL_POINTER;
        if (misaligned(partials_bf16[i], kAlign)) return EQUARX_MISALIGNED;
        mem.reads(partials_bf16[i], row_bytes(rows, cols, cols), kInPlace);
        tab.x[i] = static_cast<const uint16_t *>(partials_bf16[i]);
    }
    for (int32_t i = P; i < kMaxPartials; ++i) tab.x[i] = tab.x[i - P];
    if (int st = check_norm(residual_bf16, residual_stride, weight_bf16, rows, cols, eps, flags, outputs, mem)) return st;
    const Inputs in = inputs_of(residual_bf16, residual_stride, weight_bf16, eps, flags);
    const Outputs to = outputs_of(*outputs);
    switch (block) {
    case 32: launch_reduced<32>(tab, P, rows, cols, in, to, ctx); break;
    case 64: launch_reduced<64>(tab, P, rows, cols, in, to, ctx); break;
    case 128: launch_reduced<128>(tab, P, rows, cols, in, to, ctx); break;
    case 256: launch_reduced<256>(tab, P, rows, cols, in, to, ctx); break;
    default: launch_reduced<512>(tab, P, rows, cols, in, to, ctx); break;
    }
    return ctx.status();
}

}  // extern "C"
