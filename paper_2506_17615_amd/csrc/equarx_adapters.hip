// Host side of the adapters: argument validation, how a call is cut, and launch.
#include "equarx.h"

#include "equarx_adapters.hpp"
#include "equarx_launch.hpp"

namespace {

using namespace equarx;
using namespace equarx::host;
using namespace equarx::adapters;

constexpr int64_t kMostRows = (int64_t)1 << 24, kMostCols = (int64_t)1 << 22, kMostElements = (int64_t)1 << 40;

struct Sizes {
    int64_t M, N, K;
    int32_t rank, slices, adapters;
};

int check_sizes(const Sizes &z)
{
    if (z.M < 0 || z.N < 0 || z.K < 0 || z.M > kMostRows || z.N > kMostCols || z.K > kMostCols) return EQUARX_BAD_SHAPE;
    if (z.rank < 8 || z.rank % 8 != 0 || z.rank > EQUARX_ADAPTERS_MAX_RANK || z.slices < 1 || z.slices > EQUARX_ADAPTERS_MAX_SLICES ||
        z.adapters < 1 || z.adapters > EQUARX_ADAPTERS_MAX)
        return EQUARX_BAD_SHAPE;
    const int64_t R = (int64_t)z.rank * z.slices;
    if (z.K > kMostElements / (R * z.adapters) || z.N > kMostElements / ((int64_t)z.rank * z.adapters)) return EQUARX_BAD_SHAPE;
    return EQUARX_OK;
}

int check_rows(int64_t rows, int64_t cols, int64_t stride)
{
    return stride < cols || stride > kMostElements / rows ? EQUARX_BAD_SHAPE : EQUARX_OK;
}

inline size_t row_bytes(int64_t rows, int64_t cols, int64_t stride) { return (size_t)((rows - 1) * stride + cols) * 2; }

// How a call is cut, by its sizes alone.
struct Cut {
    Find find;              // how those who take the items have them
    bool half;              // an item of many rows is two workgroups'
    bool few_of_each;       // many items of few rows: what counts is reading A
    int tile;               // rows of an item, at most
    int64_t items;          // at most
    int32_t together;       // items of one XCD that follow each other
    int32_t rank_tiles, piece, splits, columns, chunks;
    size_t order, list, bytes;              // of the workspace: t from 0 on
};

// Rows that are taken together, rows of A and waves of a workgroup; kParts workgroups have an item's rows.
struct FewRows {
    static constexpr int RT = 1, QT = 1, W = 8, kParts = 1;
};
// Where there are workgroups enough, of items of few rows that share none of A, more rows of A to one of x: 256 rows of 200 adapters of rank 16 39.4 ->
// 35.2 us, 64 of 32 of rank 64 28.8 -> 25.9, 4096 of 200 93.5 -> 88.1; with fewer workgroups it loses (1 row 7.6 -> 8.3, 128 of 32 16.4 -> 17.1), and with many rows
// of an adapter (512 of 4 of rank 64 23.3 -> 24.3).
struct FewOfEach {
    static constexpr int RT = 1, QT = 3, W = 8, kParts = 1;
};
// Half of an item's rows, where the workgroups are at most half as many as CUs, so that k is cut in two at least: us by 64 rows -> by 32: 2048 rows of 4 adapters,
// 64 x 5376, 29.0 -> 27.1, 3000 of one 31.6 -> 28.6, 2048 of 16, two slices of 32 x 2048, 20.3 -> 17.4; in fewer pieces it loses (2048 of 64 47.3 -> 53.0,
// 3500 of 16 43.2 -> 48.1).  It is so with 4096 rows and 64 adapters at most, whose rows are found.
struct HalfMany {
    static constexpr int RT = 2, QT = 4, W = 8, kParts = 2;
};
struct ManyRows {
    static constexpr int RT = 4, QT = 4, W = 8, kParts = 1;
};

// Rows of one adapter are taken sixteen together, or 64, which reads A and B for more of them and leaves fewer workgroups.  Measured on MI355X, us by
// sixteen -> by 64, 5376 to 8192 columns, R rows of A: R = 192, 1024 rows of 4 adapters 32.4 -> 30.0, of 32 60.4 -> 49.5, of 64 68.3 -> 62.9, of 100 81.7 -> 100,
// 512 of 32 34.9 -> 34.3; R = 64, 1024 of 16 23.7 -> 22.8, of 64 38.2 -> 34.1, 512 of one 16.5 -> 18.7; R = 48, 1024 of 4 19.8 -> 21.4, 2048 of 8 30.5 -> 27.8, of 64
// 47.3 -> 42.7, of 100 53.5 either way; R = 16, 2048 of one 21.4 -> 21.9, of 64 25.0 -> 31.4, of 100 26.9 -> 38.4, 4096 of 16 45.5 -> 39.4, of 128 52.6 -> 50.9.
// k is cut where that gives more workgroups, as far as one for every CU: a workgroup of many rows has its CU's LDS for itself (one more than 256
// is a round more: 4096 rows of 4 adapters 15.6 -> 22.6); of few a second one gains nothing (64 rows 12.8, with twice as many 13.6), and what is cut
// has to be joined again (more than four pieces: 64 rows of 4 adapters of rank 16 12.9 -> 14.6).
// Items are found by those who take them, which saves the launch that lists them (333 rows 15.4 -> 13.0 us, 4096 of 4 adapters 42.6 -> 39.9, of 200
// 97.4 -> 94.4); more than 4096 rows only where no workgroup waits for another (6000 rows 32.9 -> 28.7; 8192 of 64 adapters, three such rounds, 68 -> 72).
// Few rows, without barriers, an item a row: 64 rows of 64 adapters of rank 64 49.9 -> 30.1, 128 of 200 of rank 16 32.5 -> 21.8; of few adapters the many
// workgroups of no item cost more (64 rows of 4 of rank 64 14.7 -> 21.7, 128 of 32 31.7 -> 38.9; 48 of 8 still 16.5 -> 14.6).
// Items of an XCD that follow each other: as many as an adapter has in the mean, and by sixteen half a one more, since its last is seldom full.  With
// an eighth of all for each XCD, what is left empty at the end was the last ones' (1024 rows of 200 adapters 65.2 -> 53.0 us, 8192 158 -> 124, 333 of rank
// 64 116 -> 102); without the half 1024 of 32 of rank 64 60.4 -> 63.2, with it by 64 2048 of 8 27.7 -> 29.2.
// Columns: two workgroups of the second launch for every CU (64 rows 13.2 us, with four 14.3; 4096 42.3 -> 44.2 as the rows were still listed).  From 20 Mi
// outputs on these go past the caches (4096 x 5376 44.2 -> 42.3, 4096 x 8192 58.0 -> 55.0; 2048 x 8192 34.7 -> 37.5; of 200 adapters 4096 x 8192 102 -> 98).
constexpr int64_t kTallRows = 2048, kHighRank = 64, kWorkgroupsOfFew = 256, kWorkgroupsOfMany = 256, kMostSplits = 4, kWorkgroupsOfColumns = 512,
                  kStreamFrom = (int64_t)20 << 20;

Cut cut_of(const Sizes &z)
{
    Cut c{};
    const int64_t R = (int64_t)z.rank * z.slices, groups = z.M < z.adapters ? z.M : z.adapters;
    const int64_t rows_of_each = R >= kHighRank ? 16 : R >= 48 || z.M >= 4096 ? 32 : 64;
    const bool tall = z.M >= rows_of_each * groups && z.M >= (R >= kHighRank ? kTallRows / 2 : kTallRows) && z.N >= 8;
    const bool few = z.M <= kFewRows && (z.M <= 24 || (z.M <= 64 ? 6 : 2) * groups >= z.M);
    c.tile = 16 * (tall ? ManyRows::RT : FewRows::RT);
    c.items = few ? z.M : (z.M / c.tile + groups + 7) / 8 * 8;
    c.together = (int32_t)((2 * z.M + (tall ? 2 : 3) * groups * c.tile - 1) / (2 * groups * c.tile));
    c.few_of_each = z.M < 32 * groups && (z.M / 16 + groups) * ((R + 15) / 16) >= kWorkgroupsOfFew;
    const int rank_tile = 16 * (tall ? ManyRows::QT : c.few_of_each ? FewOfEach::QT : FewRows::QT), waves = 8;
    c.rank_tiles = (int32_t)((R + rank_tile - 1) / rank_tile);
    c.half = tall && HalfMany::kParts * c.items * c.rank_tiles <= kWorkgroupsOfMany / 2;
    const int64_t steps = (z.K + kStep - 1) / kStep;
    auto limited = [](int64_t v, int64_t hi) { return v < 1 ? 1 : v < hi ? v : hi; };
    const int64_t busy = tall ? c.items * c.rank_tiles * (c.half ? HalfMany::kParts : 1) : (z.M / c.tile + groups) * c.rank_tiles;
    const int64_t splits = limited(tall ? kWorkgroupsOfMany / busy : (kWorkgroupsOfFew + busy / 2) / busy, limited((steps + waves - 1) / waves, kMostSplits));
    c.piece = (int32_t)((steps + splits - 1) / splits * kStep);
    c.splits = (int32_t)((z.K + c.piece - 1) / c.piece);
    const bool long_found = tall && busy * c.splits <= kWorkgroupsOfMany;
    c.find = few ? kFew : z.adapters > kFoundAdapters ? kListed : z.M <= kFound * 64 * waves ? kFound : long_found && z.M <= kFoundLong * 64 * waves ? kFoundLong : kListed;
    // columns of a workgroup: as many as leave enough workgroups
    c.columns = tall ? 64 : 64 * kFewWaves;
    c.chunks = (int32_t)limited((c.items * ((z.N + c.columns - 1) / c.columns) + kWorkgroupsOfColumns - 1) / kWorkgroupsOfColumns, 16);
    // Room for the partial sums of this many rows or fewer: m rows in s > 1 splits have s <= 4 / 3 * kWorkgroups / (m / 64).
    const int64_t bound = 64 * 2 * (kWorkgroupsOfFew > kWorkgroupsOfMany ? kWorkgroupsOfFew : kWorkgroupsOfMany), cut_rows = z.M * kMostSplits;
    const int64_t rows = z.M > (cut_rows < bound ? cut_rows : bound) ? z.M : (cut_rows < bound ? cut_rows : bound);
    c.order = round_up((size_t)(rows * R) * sizeof(float), kWorkspaceAlign);
    // items of sixteen rows, or of 64 and fewer
    const int64_t most_items = z.M / 16 + groups + kFewRows + 8;
    c.list = c.order + round_up((size_t)(z.M + 64 * (groups + 8) + 16 * kFewRows) * sizeof(int32_t), kWorkspaceAlign);
    c.bytes = c.list + round_up((size_t)most_items * sizeof(Item), kWorkspaceAlign);
    return c;
}

template <typename S, Find kFind>
void launch(const Sizes &z, const Cut &c, const uint16_t *x, int64_t x_stride, const uint16_t *a, const uint16_t *b, const float *factors,
            const int32_t *ids, const Slices &cut, uint16_t *out, int64_t out_stride, uint8_t *workspace, LaunchCtx &ctx)
{
    float *const t = reinterpret_cast<float *>(workspace);
    int32_t *const order = reinterpret_cast<int32_t *>(workspace + c.order);
    Item *const items = reinterpret_cast<Item *>(workspace + c.list);
    const int32_t R = z.rank * z.slices;
    if (kFind == kListed) ctx.launch(group_kernel, 1, 1024, ids, z.M, z.adapters, c.tile, order, items, c.items);
    ctx.launch3d(shrink_kernel<S::RT, S::QT, S::W, S::kParts, kFind>, (unsigned)(c.items * S::kParts), (unsigned)c.rank_tiles, (unsigned)c.splits, 64 * S::W, x, x_stride, a,
                 t, z.M, z.K, R, c.piece, order, items, ids, z.adapters, c.together * S::kParts);
    const Expansion p{out, out_stride, b, factors, t, (int32_t)z.M, (int32_t)z.N, z.rank, z.slices, c.splits, c.chunks, c.together, order, items, cut};
    auto expand = [&](auto kernel) { ctx.launch2d(kernel, (unsigned)c.items, (unsigned)cut.first_chunk[z.slices], 256, p); };
    const bool streams = z.M * z.N >= kStreamFrom;
    if constexpr (S::RT * S::kParts > 1) {
        if (streams) {
            expand(z.rank <= 32 ? expand_many_kernel<1, true> : z.rank <= 64 ? expand_many_kernel<2, true> : expand_many_kernel<4, true>);
        } else {
            expand(z.rank <= 32 ? expand_many_kernel<1, false> : z.rank <= 64 ? expand_many_kernel<2, false> : expand_many_kernel<4, false>);
        }
    } else if (kFind != kFew && streams && z.N >= 8) {
        expand(z.rank <= 32   ? expand_few_kernel<1, false, false, true>
               : z.rank <= 64 ? expand_few_kernel<2, false, false, true>
                              : expand_few_kernel<4, false, false, true>);
    } else {
        expand(z.N < 8        ? expand_few_kernel<4, kFind == kFew, true, false>
               : z.rank <= 32 ? expand_few_kernel<1, kFind == kFew, false, false>
               : z.rank <= 64 ? expand_few_kernel<2, kFind == kFew, false, false>
                              : expand_few_kernel<4, kFind == kFew, false, false>);
    }
}

}  // namespace

extern "C" {

size_t equarx_adapters_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t rank, int32_t slices, int32_t adapters)
{
    const Sizes z{M, N, K, rank, slices, adapters};
    if (check_sizes(z) != EQUARX_OK || M == 0 || N == 0 || K == 0) return 0;
    return cut_of(z).bytes;
}

int equarx_adapters(const void *x_bf16, int64_t x_stride, const void *a_bf16, const void *b_bf16, const float *factors, int32_t adapters,
                    int32_t rank, const int32_t *ids, int64_t M, int64_t N, int64_t K, const int64_t *slice_ends, int32_t slices,
                    void *out_bf16, int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    LaunchCtx ctx(stream);
    const Sizes z{M, N, K, rank, slices, adapters};
    if (int st = check_sizes(z)) return st;
    if (!slice_ends) return EQUARX_NULL_POINTER;
    for (int32_t s = 0; s < slices; ++s) {
        if (slice_ends[s] < (s == 0 ? 0 : slice_ends[s - 1]) || slice_ends[s] > N || (s + 1 == slices && slice_ends[s] != N)) return EQUARX_BAD_SHAPE;
    }
    if (M == 0 || N == 0) return EQUARX_OK;
    if (int st = check_rows(M, N, out_stride)) return st;
    if (int st = check_rows(M, K, x_stride)) return st;
    if (!out_bf16 || !factors || !ids || !b_bf16 || (K > 0 && (!x_bf16 || !a_bf16))) return EQUARX_NULL_POINTER;
    if (misaligned(x_bf16, kAlign) || misaligned(a_bf16, kAlign) || misaligned(b_bf16, kAlign) || misaligned(out_bf16, kAlign) ||
        misaligned(factors, 4) || misaligned(ids, 4) || misaligned(workspace, kWorkspaceAlign))
        return EQUARX_MISALIGNED;
    const Cut c = K > 0 ? cut_of(z) : Cut{};
    if (K > 0) {
        if (!workspace) return EQUARX_NULL_POINTER;
        if (workspace_bytes < c.bytes) return EQUARX_WORKSPACE_TOO_SMALL;
    }
    Aliasing mem;
    const size_t many = (size_t)adapters * rank;
    if (K > 0) mem.reads(x_bf16, row_bytes(M, K, x_stride));
    mem.reads(a_bf16, many * slices * (size_t)K * 2);
    mem.reads(b_bf16, many * (size_t)N * 2);
    mem.reads(factors, (size_t)adapters * sizeof(float));
    mem.reads(ids, (size_t)M * sizeof(int32_t));
    mem.writes(out_bf16, row_bytes(M, N, out_stride));
    if (K > 0) mem.writes(workspace, c.bytes);
    if (int st = mem.check()) return st;
    if (K == 0) return EQUARX_OK;
    Slices cut{};
    const int64_t width = (int64_t)c.chunks * c.columns;
    for (int32_t s = 0; s < slices; ++s) {
        const int64_t columns = slice_ends[s] - (s == 0 ? 0 : slice_ends[s - 1]);
        cut.first_column[s + 1] = (int32_t)slice_ends[s];
        cut.first_chunk[s + 1] = cut.first_chunk[s] + (int32_t)((columns + width - 1) / width);
    }
    auto pick = [&](auto shape) {
        using S = decltype(shape);
        if constexpr (S::RT * S::kParts == 1) {
            if (c.find == kFew) return launch<S, kFew>;
        } else {
            if (c.find == kFoundLong) return launch<S, kFoundLong>;
        }
        return c.find == kFound ? launch<S, kFound> : launch<S, kListed>;
    };
    auto *const go = c.half ? launch<HalfMany, kFound> : c.tile != 16 ? pick(ManyRows{}) : c.few_of_each ? pick(FewOfEach{}) : pick(FewRows{});
    go(z, c, static_cast<const uint16_t *>(x_bf16), x_stride, static_cast<const uint16_t *>(a_bf16), static_cast<const uint16_t *>(b_bf16), factors, ids,
       cut, static_cast<uint16_t *>(out_bf16), out_stride, static_cast<uint8_t *>(workspace), ctx);
    return ctx.status();
}

}  // extern "C"
