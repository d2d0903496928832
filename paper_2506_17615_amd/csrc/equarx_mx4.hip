// Host side of the 4-bit microscaled calls: argument validation, kernel selection and launch.
#include "equarx.h"

#include "equarx_launch.hpp"
#include "equarx_mx4.hpp"

namespace {

using namespace equarx;
using namespace equarx::host;
using namespace equarx::mx4;

constexpr int64_t kMostRows = INT32_MAX;

inline int64_t groups_of(int64_t cols) { return (cols + kGroup - 1) / kGroup; }

// A row-major tensor's shape; one that holds nothing may have any stride.
int check_rows(int64_t rows, int64_t cols, int64_t stride)
{
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostRows) return EQUARX_BAD_SHAPE;
    if (rows == 0 || cols == 0) return EQUARX_OK;
    if (stride < cols || stride > ((int64_t)1 << 40) / rows || groups_of(cols) * kGroup > ((int64_t)1 << 40) / rows)
        return EQUARX_BAD_SHAPE;
    return EQUARX_OK;
}

inline size_t row_bytes(int64_t rows, int64_t cols, int64_t stride) { return (size_t)((rows - 1) * stride + cols) * 2; }
inline size_t code_bytes(int64_t rows, int64_t cols) { return (size_t)(rows * groups_of(cols)) * (kGroup / 2); }
inline size_t scale_bytes(int64_t rows, int64_t cols) { return (size_t)(rows * groups_of(cols)) * (kGroup / kBlock); }

// f(first row, rows) in pieces whose units of eight elements can be counted in 31 bits.
template <typename F>
void in_row_pieces(int64_t rows, int64_t cols, F f)
{
    const int64_t row_units = groups_of(cols) * 16;
    const int64_t most = ((int64_t)1 << 30) / row_units;        // at least 4: a row has fewer than 2^28 units
    for (int64_t at = 0; at < rows; at += most) f(at, rows - at < most ? rows - at : most);
}

void launch_quantize_rows(const uint16_t *x, int64_t rows, int64_t cols, int64_t x_stride, uint8_t *codes, uint8_t *scales,
                          LaunchCtx &ctx)
{
    const int64_t groups = groups_of(cols);
    const Divisor row_units((uint32_t)(groups * 16));
    in_row_pieces(rows, cols, [&](int64_t at, int64_t count) {
        const uint32_t units = (uint32_t)(count * groups * 16);
        ctx.launch(quantize_rows_kernel, (units + 255) / 256, 256, x + at * x_stride, x_stride, codes + at * groups * 64,
                   scales + at * groups * 4, cols, units, row_units);
    });
}

// A product's operands: x packed, or bf16 rows that the kernel packs (x_scales is then null and x_stride counts).
struct Product {
    const uint8_t *xc, *xs, *wc, *ws;
    uint16_t *out;
    int64_t M, N, K, out_stride, x_stride;
};

// Does a workgroup of the kernel for few rows pack x itself?
inline bool packs_itself(int64_t M, int64_t K) { return M <= kMostQuantizedRows && M * groups_of(K) * kGroup <= kMostQuantized; }

constexpr int64_t kPieceN = (int64_t)1 << 26;           // rows of w in one launch, at most

template <int WN, int WM, int FN, int FM, int kBuffers>
void launch_tiles(const Product &p, LaunchCtx &ctx)
{
    constexpr int64_t kN = WN * FN * 32, kM = WM * FM * 32;
    const int64_t groups = groups_of(p.K);
    for (int64_t n = 0; n < p.N; n += kPieceN) {
        const int64_t N = p.N - n < kPieceN ? p.N - n : kPieceN, tiles_n = (N + kN - 1) / kN;
        const int64_t most = (kGridThreads / (64 * WN * WM)) / tiles_n * kM;    // rows of x in one launch: 31 tiles at least
        for (int64_t at = 0; at < p.M; at += most) {
            const int64_t m = p.M - at < most ? p.M - at : most, tiles_m = (m + kM - 1) / kM;
            ctx.launch(product_tiles_kernel<WN, WM, FN, FM, kBuffers>, (unsigned)(tiles_n * tiles_m), 64 * WN * WM,
                       p.xc + at * groups * 64, p.xs + at * groups * 4, p.wc + n * groups * 64, p.ws + n * groups * 4,
                       p.out + at * p.out_stride + n, (int32_t)m, (int32_t)N, (int32_t)groups, p.out_stride, (uint32_t)tiles_n,
                       (uint32_t)tiles_m);
        }
    }
}

template <int MT, bool kQuantize>
void launch_rows(const Product &p, LaunchCtx &ctx)
{
    const int64_t groups = groups_of(p.K);
    constexpr int64_t kPieceM = (int64_t)32768 * 32 * MT;       // rows of x in one launch
    for (int64_t n = 0; n < p.N; n += kPieceN) {
        const int64_t N = p.N - n < kPieceN ? p.N - n : kPieceN;
        for (int64_t m = 0; m < p.M; m += kPieceM) {
            const int64_t M = p.M - m < kPieceM ? p.M - m : kPieceM;
            ctx.launch2d(product_rows_kernel<MT, kQuantize>, (unsigned)((N + 31) / 32), (unsigned)((M + 32 * MT - 1) / (32 * MT)),
                         256, kQuantize ? p.xc : p.xc + m * groups * 64, kQuantize ? p.xs : p.xs + m * groups * 4,
                         p.wc + n * groups * 64, p.ws + n * groups * 4, p.out + m * p.out_stride + n, (int32_t)M, (int32_t)N,
                         (int32_t)groups, p.out_stride, p.x_stride, (int32_t)p.K);
        }
    }
}

// Which kernel takes a product.  Up to 64 rows of x: the one for few rows.  Above, the smallest tile whose workgroups the chip's 256
// CUs hold at once, one each, since a workgroup alone on its CU waits for loads more than for anything; with more workgroups
// than that 128 x 128 with two on a CU, or 256 x 256, by the rounds they make, whole rounds and part ones (the mean of the
// two), of 0.70 and 1.09 us a group of k.  Measured on MI355X, us (w rows n x x rows m; products of N x K):
//                           128 x 64    128 x 128     two a CU
//     M     N x K           32 x 128     4 buffers     2 buffers   256 x 256
//     96    5376 x 5376     10.4   12.3     16.0          19.5       30.7
//     192                   19.8   12.9     17.0          20.3       32.8
//     333                   21.4   14.5     17.7          21.2       34.0
//     512                   30.7   24.9     19.3          22.3       34.4
//     1024                   --    39.5     36.0          29.0       37.8
//     2048                   --    76.6     59.7          51.7       44.6
//     192   2560 x 8192     14.0   15.7     22.2          27.9       43.6
//     512                   27.5   16.6     22.8          28.5       45.3
//     1024                   --    31.5     24.3          29.5       46.1
//     2048                   --    46.9     47.0          38.8       48.7
//     192   8192 x 1024      9.7    5.3      6.6           6.2       11.4
//     512                   20.0    9.5      7.7           7.5       12.8
//     1024                   --    17.4     13.5          11.8       14.7
//     2048                   --    32.3     24.7          19.6       16.9
//     8192  8192 x 8192                                    363        279
// Fewer than four groups of k have their scales loaded one by one, which only the kernel for few rows does.
constexpr int64_t kCUs = 256;

void launch_product(const Product &p, LaunchCtx &ctx)
{
    const int64_t groups = groups_of(p.K);
    auto tiles = [&](int64_t n, int64_t m) { return ((p.N + n - 1) / n) * ((p.M + m - 1) / m); };
    auto rounds = [](int64_t t, int64_t at_once) { return (double)t / at_once + (double)((t + at_once - 1) / at_once); };
    if (p.M <= 32) {
        if (p.xs || groups == 0) {
            launch_rows<1, false>(p, ctx);
        } else {
            launch_rows<1, true>(p, ctx);
        }
    } else if (p.M <= 64) {
        launch_rows<2, false>(p, ctx);
    } else if (groups < 4 || tiles(32, 128) <= kCUs) {
        launch_rows<4, false>(p, ctx);
    } else if (tiles(128, 64) <= kCUs) {
        launch_tiles<2, 2, 2, 1, 4>(p, ctx);
    } else if (tiles(128, 128) <= kCUs) {
        launch_tiles<2, 2, 2, 2, 4>(p, ctx);
    } else if (rounds(tiles(128, 128), 2 * kCUs) * 0.70 < rounds(tiles(256, 256), kCUs) * 1.09) {
        launch_tiles<2, 2, 2, 2, 2>(p, ctx);
    } else {
        launch_tiles<2, 2, 4, 4, 2>(p, ctx);
    }
}

// The workspace of a linear call: x's codes, and from `scales` on its scales; none where the product's kernel packs x.
struct Workspace {
    size_t scales, bytes;
};

Workspace plan_workspace(int64_t M, int64_t K)
{
    Workspace w{};
    if (K == 0 || packs_itself(M, K)) return w;
    w.scales = round_up(code_bytes(M, K), kWorkspaceAlign);
    w.bytes = w.scales + round_up(scale_bytes(M, K), kWorkspaceAlign);
    return w;
}

int check_product(int64_t M, int64_t N, int64_t K, int64_t out_stride)
{
    if (M < 0 || N < 0 || K < 0 || M > kMostRows || N > kMostRows || K > kMostK) return EQUARX_BAD_SHAPE;
    if (int st = check_rows(M, N, out_stride)) return st;
    if (int st = check_rows(M, K, K)) return st;
    return check_rows(N, K, K);
}

}  // namespace

extern "C" {

int64_t equarx_mx4_row_blocks(int64_t cols)
{
    return cols < 0 || cols > kMostRows ? 0 : groups_of(cols) * (kGroup / kBlock);
}

int equarx_mx4_quantize(const void *x_bf16, int64_t rows, int64_t cols, int64_t x_stride, uint8_t *codes, uint8_t *scales,
                        void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_rows(rows, cols, x_stride)) return st;
    if (rows == 0 || cols == 0) return EQUARX_OK;
    if (!x_bf16 || !codes || !scales) return EQUARX_NULL_POINTER;
    if (misaligned(x_bf16, kAlign) || misaligned(codes, kAlign) || misaligned(scales, kAlign)) return EQUARX_MISALIGNED;
    Aliasing mem;
    mem.reads(x_bf16, row_bytes(rows, cols, x_stride));
    mem.writes(codes, code_bytes(rows, cols));
    mem.writes(scales, scale_bytes(rows, cols));
    if (int st = mem.check()) return st;
    launch_quantize_rows(static_cast<const uint16_t *>(x_bf16), rows, cols, x_stride, codes, scales, ctx);
    return ctx.status();
}

int equarx_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out_bf16,
                          int64_t out_stride, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_rows(rows, cols, out_stride)) return st;
    if (rows == 0 || cols == 0) return EQUARX_OK;
    if (!codes || !scales || !out_bf16) return EQUARX_NULL_POINTER;
    if (misaligned(codes, kAlign) || misaligned(scales, kAlign) || misaligned(out_bf16, kAlign)) return EQUARX_MISALIGNED;
    Aliasing mem;
    mem.reads(codes, code_bytes(rows, cols));
    mem.reads(scales, scale_bytes(rows, cols));
    mem.writes(out_bf16, row_bytes(rows, cols, out_stride));
    if (int st = mem.check()) return st;
    const int64_t groups = groups_of(cols);
    const Divisor row_units((uint32_t)(groups * 16));
    in_row_pieces(rows, cols, [&](int64_t at, int64_t count) {
        const uint32_t units = (uint32_t)(count * groups * 16);
        ctx.launch(dequantize_rows_kernel, (units + 255) / 256, 256, codes + at * groups * 64, scales + at * groups * 4,
                   static_cast<uint16_t *>(out_bf16) + at * out_stride, out_stride, cols, units, row_units);
    });
    return ctx.status();
}

size_t equarx_mx4_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (check_product(M, N, K, N) != EQUARX_OK || M == 0 || N == 0 || K == 0) return 0;
    return plan_workspace(M, K).bytes;
}

int equarx_mx4_product(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes, const uint8_t *w_scales,
                       int64_t M, int64_t N, int64_t K, void *out_bf16, int64_t out_stride, void * /*workspace*/,
                       size_t /*workspace_bytes*/, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_product(M, N, K, out_stride)) return st;
    if (M == 0 || N == 0) return EQUARX_OK;
    if (!out_bf16) return EQUARX_NULL_POINTER;
    if (K > 0 && (!x_codes || !x_scales || !w_codes || !w_scales)) return EQUARX_NULL_POINTER;
    if (misaligned(out_bf16, kAlign) || misaligned(x_codes, kAlign) || misaligned(x_scales, kAlign) ||
        misaligned(w_codes, kAlign) || misaligned(w_scales, kAlign))
        return EQUARX_MISALIGNED;
    Aliasing mem;
    mem.reads(x_codes, code_bytes(M, K));
    mem.reads(x_scales, scale_bytes(M, K));
    mem.reads(w_codes, code_bytes(N, K));
    mem.reads(w_scales, scale_bytes(N, K));
    mem.writes(out_bf16, row_bytes(M, N, out_stride));
    if (int st = mem.check()) return st;
    launch_product({x_codes, x_scales, w_codes, w_scales, static_cast<uint16_t *>(out_bf16), M, N, K, out_stride, 0}, ctx);
    return ctx.status();
}

int equarx_mx4_linear(const void *x_bf16, int64_t x_stride, const uint8_t *w_codes, const uint8_t *w_scales, int64_t M,
                      int64_t N, int64_t K, void *out_bf16, int64_t out_stride, void *workspace, size_t workspace_bytes,
                      void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_product(M, N, K, out_stride)) return st;
    if (int st = check_rows(M, K, x_stride)) return st;
    if (M == 0 || N == 0) return EQUARX_OK;
    if (!out_bf16) return EQUARX_NULL_POINTER;
    if (K > 0 && (!x_bf16 || !w_codes || !w_scales)) return EQUARX_NULL_POINTER;
    if (misaligned(out_bf16, kAlign) || misaligned(x_bf16, kAlign) || misaligned(w_codes, kAlign) ||
        misaligned(w_scales, kAlign) || misaligned(workspace, kWorkspaceAlign))
        return EQUARX_MISALIGNED;
    const Workspace plan = plan_workspace(M, K);
    const size_t need = plan.bytes;
    if (need > 0 && !workspace) return EQUARX_NULL_POINTER;
    if (workspace_bytes < need) return EQUARX_WORKSPACE_TOO_SMALL;
    Aliasing mem;
    if (K > 0) mem.reads(x_bf16, row_bytes(M, K, x_stride));
    mem.reads(w_codes, code_bytes(N, K));
    mem.reads(w_scales, scale_bytes(N, K));
    mem.writes(out_bf16, row_bytes(M, N, out_stride));
    mem.writes(workspace, need);
    if (int st = mem.check()) return st;
    uint8_t *const codes = static_cast<uint8_t *>(workspace);
    uint8_t *const scales = codes ? codes + plan.scales : nullptr;
    Product p{codes, scales, w_codes, w_scales, static_cast<uint16_t *>(out_bf16), M, N, K, out_stride, x_stride};
    if (packs_itself(M, K)) {
        p.xc = static_cast<const uint8_t *>(x_bf16);
        p.xs = nullptr;
    } else if (K > 0) {
        launch_quantize_rows(static_cast<const uint16_t *>(x_bf16), M, K, x_stride, codes, scales, ctx);
    }
    launch_product(p, ctx);
    return ctx.status();
}

}  // extern "C"
