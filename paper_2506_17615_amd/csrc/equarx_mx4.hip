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

void launch_product(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, int64_t M, int64_t N,
                    int64_t K, uint16_t *out, int64_t out_stride, LaunchCtx &ctx)
{
    const int32_t groups = (int32_t)groups_of(K);
    if (M > 64 && groups >= 4 && groups <= kMostTileGroups) {
        const uint32_t tiles_n = (uint32_t)((N + 255) / 256), tiles_m = (uint32_t)((M + 255) / 256);
        ctx.launch(product_tiles_kernel<2, 2, 4, 4>, tiles_n * tiles_m, 256, xc, xs, wc, ws, out, (int32_t)M, (int32_t)N, groups,
                   out_stride, tiles_n, tiles_m);
        return;
    }
    const int64_t piece = 65535 * 64;                           // rows of x in one launch: the grid's second dimension
    for (int64_t at = 0; at < M; at += piece) {
        const int64_t m = M - at < piece ? M - at : piece;
        ctx.launch2d(product_rows_kernel<4, 4>, (unsigned)((N + 15) / 16), (unsigned)((m + 63) / 64), 256,
                     xc + at * groups * 64, xs + at * groups * 4, wc, ws, out + at * out_stride, (int32_t)m, (int32_t)N,
                     groups, out_stride);
    }
}

// The parts of a workspace: x's codes and scales where the call quantizes x itself.
struct Workspace {
    size_t codes, scales, bytes;
};

Workspace plan_workspace(int64_t M, int64_t K)
{
    Workspace w;
    w.codes = 0;
    w.scales = round_up(code_bytes(M, K), kWorkspaceAlign);
    w.bytes = w.scales + round_up(scale_bytes(M, K), kWorkspaceAlign);
    return w;
}

int check_product(int64_t M, int64_t N, int64_t K, int64_t out_stride)
{
    if (M < 0 || N < 0 || K < 0 || M > kMostRows || N > kMostRows || K > kMostRows) return EQUARX_BAD_SHAPE;
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
                       int64_t M, int64_t N, int64_t K, void *out_bf16, int64_t out_stride, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_product(M, N, K, out_stride)) return st;
    if (M == 0 || N == 0) return EQUARX_OK;
    if (!out_bf16) return EQUARX_NULL_POINTER;
    if (K > 0 && (!x_codes || !x_scales || !w_codes || !w_scales)) return EQUARX_NULL_POINTER;
    if (misaligned(out_bf16, kAlign) || misaligned(x_codes, kAlign) || misaligned(x_scales, kAlign) ||
        misaligned(w_codes, kAlign) || misaligned(w_scales, kAlign) || misaligned(workspace, kWorkspaceAlign))
        return EQUARX_MISALIGNED;
    const size_t need = K > 0 ? plan_workspace(M, K).bytes : 0;
    if (need > 0 && !workspace) return EQUARX_NULL_POINTER;
    if (workspace_bytes < need) return EQUARX_WORKSPACE_TOO_SMALL;
    Aliasing mem;
    mem.reads(x_codes, code_bytes(M, K));
    mem.reads(x_scales, scale_bytes(M, K));
    mem.reads(w_codes, code_bytes(N, K));
    mem.reads(w_scales, scale_bytes(N, K));
    mem.writes(out_bf16, row_bytes(M, N, out_stride));
    mem.writes(workspace, need);
    if (int st = mem.check()) return st;
    launch_product(x_codes, x_scales, w_codes, w_scales, M, N, K, static_cast<uint16_t *>(out_bf16), out_stride, ctx);
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
    const size_t need = K > 0 ? plan.bytes : 0;
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
    if (K > 0) launch_quantize_rows(static_cast<const uint16_t *>(x_bf16), M, K, x_stride, codes, scales, ctx);
    launch_product(codes, scales, w_codes, w_scales, M, N, K, static_cast<uint16_t *>(out_bf16), out_stride, ctx);
    return ctx.status();
}

}  // extern "C"
