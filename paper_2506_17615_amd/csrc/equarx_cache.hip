// Host side of the key/value cache calls: argument validation, kernel selection and launch.
#include "equarx.h"

#include <type_traits>

#include "equarx_cache.hpp"
#include "equarx_launch.hpp"

namespace {

using namespace equarx;
using namespace equarx::host;
using namespace equarx::cache;

constexpr int64_t kMostElements = (int64_t)1 << 40;
constexpr int kGridDim = 65535;         // of a grid's second and third dimension

int check_cache(const equarx_cache *c)
{
    if (!c) return EQUARX_NULL_POINTER;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return EQUARX_BAD_SHAPE;
    if ((c->block != 64 && c->block != 128 && c->block != 256) || c->block > c->dim) return EQUARX_BAD_BLOCK;
    if (c->pages < 1 || c->heads < 1 || c->heads > kGridDim || c->page < 16 || c->page % 16 != 0 || c->page > 65536)
        return EQUARX_BAD_SHAPE;
    if (c->pages > INT32_MAX || c->pages > kMostElements / ((int64_t)c->heads * c->page * c->dim)) return EQUARX_BAD_SHAPE;
    if (!c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return EQUARX_NULL_POINTER;
    if (misaligned(c->k_codes, kAlign) || misaligned(c->k_scales, kAlign) || misaligned(c->v_codes, kAlign) ||
        misaligned(c->v_scales, kAlign))
        return EQUARX_MISALIGNED;
    return EQUARX_OK;
}

Pool pool_of(const equarx_cache &c)
{
    Pool p{c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.pages, c.heads, c.page, -1};
    for (int s = 4; s <= 16; ++s) {
        if (c.page == 1 << s) p.page_shift = s;
    }
    return p;
}

void list_cache(const equarx_cache &c, bool written, Aliasing &mem)
{
    const size_t codes = (size_t)c.pages * c.heads * c.page * c.dim, scales = codes / c.block * sizeof(float);
    const void *const parts[4] = {c.k_codes, c.v_codes, c.k_scales, c.v_scales};
    for (int i = 0; i < 4; ++i) {
        if (written) {
            mem.writes(parts[i], i < 2 ? codes : scales);
        } else {
            mem.reads(parts[i], i < 2 ? codes : scales);
        }
    }
}

// bf16 [rows][heads][dim] with strides; the bytes from its first element to its last.
int check_tokens(const void *p, int64_t rows, int64_t heads, int64_t dim, int64_t row_stride, int64_t head_stride, size_t &bytes)
{
    if (!p) return EQUARX_NULL_POINTER;
    if (misaligned(p, kAlign) || row_stride % 8 != 0 || head_stride % 8 != 0) return EQUARX_MISALIGNED;
    if (row_stride < 0 || head_stride < 0 || row_stride > kMostElements / rows || head_stride > kMostElements / heads)
        return EQUARX_BAD_SHAPE;
    bytes = (size_t)((rows - 1) * row_stride + (heads - 1) * head_stride + dim) * 2;
    return EQUARX_OK;
}

// f(dim, block) as compile-time constants.
template <typename F>
void with_geometry(int32_t dim, int32_t block, F f)
{
    using std::integral_constant;
#define EQUARX_GEOMETRY(D, B) \
    if (dim == D && block == B) f(integral_constant<int, D>{}, integral_constant<int, B>{})
    EQUARX_GEOMETRY(64, 64);
    EQUARX_GEOMETRY(128, 64);
    EQUARX_GEOMETRY(128, 128);
    EQUARX_GEOMETRY(256, 64);
    EQUARX_GEOMETRY(256, 128);
    EQUARX_GEOMETRY(256, 256);
#undef EQUARX_GEOMETRY
}

// f(first, count) in pieces whose threads a grid can hold, 256 a row at most.
template <typename F>
void in_launches(int64_t rows, F f)
{
    constexpr int64_t kPiece = (int64_t)1 << 22;
    for (int64_t at = 0; at < rows; at += kPiece) f(at, rows - at < kPiece ? rows - at : kPiece);
}

int check_sequences(const int32_t *page_table, int64_t table_width, const int32_t *lengths, int32_t sequences, Aliasing &mem)
{
    if (!page_table || !lengths) return EQUARX_NULL_POINTER;
    if (misaligned(page_table, sizeof(int32_t)) || misaligned(lengths, sizeof(int32_t))) return EQUARX_MISALIGNED;
    mem.reads(page_table, (size_t)sequences * (size_t)table_width * sizeof(int32_t));
    mem.reads(lengths, (size_t)sequences * sizeof(int32_t));
    return EQUARX_OK;
}

// ---------------------------------------------------------------- how an attention call is cut

// Sequences up to here are not shared out.
constexpr int64_t kShortest = 512;

// A call goes to one of three kernels' forms.
enum class AttentionForm { kRows, kShared, kWhole };

struct AttentionPlan {
    AttentionForm form;
    int rows16;                 // sixteens of rows of a wave
    int64_t row_tiles;          // of the longest query run
    int32_t splits, chunk;      // kRows
    bool tiles_last;
};

// A wave of the kernels for few rows holds 32 rows of heads up to 128; of 256 their sums spill: 24 rows of 8 sequences of up to 4096
// tokens, blocks of 64: 78 us, and 62 with many rows' kernel.
inline int64_t few_rows(int32_t dim) { return dim <= 128 ? 32 : 16; }

// Many rows, by workgroups of 128: as many workgroups as the CUs hold at once, two each and one with heads of 256.
inline int64_t held_at_once(int32_t dim) { return dim <= 128 ? 512 : 256; }

// Splits of the tokens for so many workgroups of rows: as many as are held at once, none with fewer than four tiles of tokens: 5
// queries of 8 heads after 131072 tokens 27 us in 256 splits, 65 in 64; twice as many workgroups, 202 for 192 us (512 queries
// of 32 heads after 16384).  No more for more workgroups, no fewer for more tokens.  All tokens are split, whatever a window lets
// rows see of them: 40 queries of 16 heads over 4 after 131072 tokens with a window of 1024 63 us, after 1088 tokens 17.
inline int64_t splits_for(int64_t workgroups, int32_t heads, int32_t dim, int64_t max_length)
{
    const int64_t held = held_at_once(dim), most = (max_length + 255) / 256;
    int64_t splits = (held + workgroups - 1) / workgroups;
    if (splits > most) splits = most;
    if (splits > 256) splits = 256;
    if (splits * heads > kGridDim) splits = kGridDim / heads;
    return splits < 1 ? 1 : splits;
}

// One form for a call, by its longest run: a chunk of 512 queries and 63 single tokens of 32 heads over 8, after up to 8192
// tokens, are 746 us in one call, where the single tokens go the way of many rows, and 131 and 100 us in two.
AttentionPlan plan_attention(int32_t heads, int32_t dim, int32_t q_heads, int32_t sequences, int64_t max_queries, int64_t max_length)
{
    AttentionPlan p{};
    const int64_t rows = max_queries * (q_heads / heads);
    p.rows16 = rows <= 16 ? 1 : 2;
    p.splits = 1;
    if (rows <= few_rows(dim)) {
        p.row_tiles = 1;
        p.form = sequences > kMostShared || max_length <= kShortest ? AttentionForm::kWhole : AttentionForm::kShared;
        return p;
    }
    p.form = AttentionForm::kRows;
    p.row_tiles = (rows + 127) / 128;
    const int64_t workgroups = p.row_tiles * heads * sequences;
    const int64_t splits = splits_for(workgroups, heads, dim, max_length);
    p.chunk = (int32_t)(((max_length + splits - 1) / splits + 63) / 64 * 64);
    p.splits = (int32_t)((max_length + p.chunk - 1) / p.chunk);
    // Long workgroups should be launched first, and a CU have long ones and short ones.  Tiles are launched longest first; where
    // their lengths differ most within a sequence, or all are held at once, tile after tile over all sequences (8 prompts of 1024
    // tokens, 16 heads of 64: 50 us for 65), else sequence after sequence (2 x 2048 queries of 32 heads of 128 after 8192 and
    // 5120 tokens: 629 us for 752).
    p.tiles_last = workgroups * p.splits <= held_at_once(dim) || max_queries * 2 > max_length;
    return p;
}

inline size_t part_bytes(int32_t dim) { return ((size_t)dim + 2) * sizeof(float); }
inline size_t shares_bytes(int rows16, int32_t dim)
{
    return (size_t)kShares * 2 * rows16 * 16 * part_bytes(dim) + (kMostShared + 1) * sizeof(int64_t);
}
inline size_t splits_bytes(int64_t splits, int64_t q_rows, int32_t q_heads, int32_t dim)
{
    return splits == 1 ? 0 : (size_t)splits * (size_t)q_rows * (size_t)q_heads * part_bytes(dim);
}

size_t attention_workspace(const AttentionPlan &p, int32_t dim, int64_t q_rows, int32_t q_heads)
{
    return p.form == AttentionForm::kShared ? shares_bytes(p.rows16, dim) : splits_bytes(p.splits, q_rows, q_heads, dim);
}

// What no call of up to so many rows, sequences and tokens needs more than, as long as its rows are at most its sequences times its
// longest run.  Fewer sequences or shorter runs may need more: fewer workgroups of rows are cut into more splits.
size_t most_attention_workspace(int32_t heads, int32_t dim, int64_t q_rows, int32_t q_heads, int32_t sequences, int64_t max_length)
{
    const int64_t group = q_heads / heads, few = few_rows(dim), held = held_at_once(dim);
    size_t most = 0;
    if (group <= few && max_length > kShortest) most = shares_bytes(few / group * group <= 16 ? 1 : 2, dim);
    for (int64_t s = 1; s <= sequences && s * heads < held; ++s) {
        // tiles of rows of the longest run, which is as long as that allows; from `held` workgroups on there is one split
        for (int64_t tiles = 1; tiles * s * heads < held; ++tiles) {
            const int64_t longest = tiles * 128 / group;
            if (longest * group <= (tiles - 1) * 128) continue;         // none of so many
            const int64_t rows = s * longest < q_rows ? s * longest : q_rows;
            const size_t bytes = splits_bytes(splits_for(tiles * s * heads, heads, dim, max_length), rows, q_heads, dim);
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

// The kernels of one geometry.
template <int D, int NB>
void launch_attention(const AttentionPlan &plan, const AttentionCall &call, const Sequences &seqs, const Pool &pool, LaunchCtx &ctx)
{
    const int64_t tiles = plan.row_tiles < kGridDim ? plan.row_tiles : kGridDim;
    const int64_t all = call.q_rows * call.q_heads;
    auto share = [&](auto rows16) {
        constexpr int R = decltype(rows16)::value;
        ctx.launch(attention_shares_kernel<D, NB, R>, (unsigned)kShares / 4, 256, call, seqs, pool);
        // many items have few parts each: a wave joins them; few have many: four
        in_launches(all, [&](int64_t first, int64_t rows) {
            if ((int64_t)call.sequences * pool.heads * 8 >= kShares) {
                ctx.launch(join_shares_kernel<D, R, 1>, (unsigned)((rows + 3) / 4), 256, call, seqs, pool, first);
            } else {
                ctx.launch(join_shares_kernel<D, R, 4>, (unsigned)rows, 256, call, seqs, pool, first);
            }
        });
    };
    if (plan.form == AttentionForm::kShared) {
        if (plan.rows16 == 1) share(std::integral_constant<int, 1>{});
        if constexpr (D <= 128) {
            if (plan.rows16 == 2) share(std::integral_constant<int, 2>{});
        }
        return;
    }
    auto tokens_kernel = attention_tokens_kernel<D, NB, 1>;
    if constexpr (D <= 128) {
        if (plan.rows16 == 2) tokens_kernel = attention_tokens_kernel<D, NB, 2>;
    }
    for (int32_t at = 0; at < call.sequences; at += kGridDim) {
        const int32_t count = call.sequences - at < kGridDim ? call.sequences - at : kGridDim;
        AttentionCall part = call;
        part.q_starts += at;
        const Sequences some{seqs.table + at * seqs.width, seqs.lengths + at, seqs.width};
        if (plan.form == AttentionForm::kRows) {
            part.tiles_last = plan.tiles_last;
            ctx.launch3d(attention_rows_kernel<D, NB>, (unsigned)(pool.heads * plan.splits), (unsigned)(plan.tiles_last ? count : tiles),
                         (unsigned)(plan.tiles_last ? tiles : count), 256, part, some, pool);
        } else {
            ctx.launch3d(tokens_kernel, (unsigned)tiles, (unsigned)pool.heads, (unsigned)count, 256, part, some, pool);
        }
    }
    if (plan.splits == 1) return;
    in_launches(all, [&](int64_t first, int64_t rows) {
        if (plan.splits > 8) {
            ctx.launch(join_splits_kernel<D, 4>, (unsigned)rows, 256, call, first);
        } else {
            ctx.launch(join_splits_kernel<D, 1>, (unsigned)((rows + 3) / 4), 256, call, first);
        }
    });
}

int check_heads(int32_t heads, int64_t q_rows, int32_t q_heads, int32_t dim, int32_t sequences, int32_t max_queries,
                int64_t max_length)
{
    if (heads < 1 || heads > kGridDim || q_heads < 1 || q_heads % heads != 0) return EQUARX_BAD_SHAPE;
    if (q_rows < 0 || sequences < 0 || max_queries < 1 || max_length < 1 || max_length > INT32_MAX - 63) return EQUARX_BAD_SHAPE;
    if (dim != 64 && dim != 128 && dim != 256) return EQUARX_BAD_SHAPE;
    if (q_rows > (INT32_MAX - 127) / q_heads) return EQUARX_BAD_SHAPE;      // a kernel rounds up to its 128 rows
    return EQUARX_OK;
}

}  // namespace

extern "C" {

int equarx_cache_write(const equarx_cache *cache, const void *k_bf16, int64_t k_row_stride, int64_t k_head_stride,
                       const void *v_bf16, int64_t v_row_stride, int64_t v_head_stride, int64_t tokens, const int64_t *slots,
                       void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_cache(cache)) return st;
    if (tokens < 0 || tokens > (1 << 30)) return EQUARX_BAD_SHAPE;
    if (tokens == 0) return EQUARX_OK;
    size_t k_bytes, v_bytes;
    if (int st = check_tokens(k_bf16, tokens, cache->heads, cache->dim, k_row_stride, k_head_stride, k_bytes)) return st;
    if (int st = check_tokens(v_bf16, tokens, cache->heads, cache->dim, v_row_stride, v_head_stride, v_bytes)) return st;
    if (!slots) return EQUARX_NULL_POINTER;
    if (misaligned(slots, sizeof(int64_t))) return EQUARX_MISALIGNED;
    Aliasing mem;
    mem.reads(k_bf16, k_bytes);
    mem.reads(v_bf16, v_bytes);
    mem.reads(slots, (size_t)tokens * sizeof(int64_t));
    list_cache(*cache, true, mem);
    if (int st = mem.check()) return st;
    with_geometry(cache->dim, cache->block, [&](auto dim, auto block) {
        constexpr int D = decltype(dim)::value, B = decltype(block)::value;
        auto with = [&](auto each) {
            constexpr int T = decltype(each)::value, kTokens = 256 / (D / 8) * T;
            in_launches(tokens, [&](int64_t at, int64_t count) {
                ctx.launch2d(write_kernel<D, B, T>, (unsigned)((count + kTokens - 1) / kTokens), (unsigned)cache->heads, 256,
                             static_cast<const uint16_t *>(k_bf16) + at * k_row_stride,
                             static_cast<const uint16_t *>(v_bf16) + at * v_row_stride, slots + at, k_row_stride, v_row_stride,
                             (int32_t)count, k_head_stride, v_head_stride, pool_of(*cache));
            });
        };
        // Four tokens a lane once that gives every CU a workgroup: 16384 tokens of 8 heads of 128 in 20 us, one a lane 43; 64
        // tokens in no order, as a decode step has them, one a lane 3.8 us, four 8 to 10.
        constexpr int kTokens = 256 / (D / 8) * 4;
        if ((tokens + kTokens - 1) / kTokens * cache->heads < 256)
            with(std::integral_constant<int, 1>{});
        else
            with(std::integral_constant<int, 4>{});
    });
    return ctx.status();
}

int equarx_cache_read(const equarx_cache *cache, const int32_t *page_table, int64_t table_width, const int32_t *lengths,
                      const int32_t *starts, int32_t sequences, int64_t max_length, int64_t rows, void *k_out, void *v_out,
                      void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_cache(cache)) return st;
    if (sequences < 0 || table_width < 0 || table_width > INT32_MAX || max_length < 0 || rows < 0 || rows > INT32_MAX ||
        rows > kMostElements / ((int64_t)cache->heads * cache->dim))
        return EQUARX_BAD_SHAPE;
    if (sequences == 0 || table_width == 0 || rows == 0) return EQUARX_OK;
    Aliasing mem;
    if (int st = check_sequences(page_table, table_width, lengths, sequences, mem)) return st;
    if (!starts || !k_out || !v_out) return EQUARX_NULL_POINTER;
    if (misaligned(starts, sizeof(int32_t)) || misaligned(k_out, kAlign) || misaligned(v_out, kAlign)) return EQUARX_MISALIGNED;
    const size_t out_bytes = (size_t)rows * cache->heads * cache->dim * 2;
    mem.reads(starts, (size_t)sequences * sizeof(int32_t));
    mem.writes(k_out, out_bytes);
    mem.writes(v_out, out_bytes);
    list_cache(*cache, false, mem);
    if (int st = mem.check()) return st;
    with_geometry(cache->dim, cache->block, [&](auto dim, auto block) {
        constexpr int D = decltype(dim)::value, B = decltype(block)::value;
        constexpr int kTokens = 256 / (D / 8) * 4;
        int64_t tiles = (max_length + kTokens - 1) / kTokens;
        tiles = tiles < 1 ? 1 : tiles < 4096 ? tiles : 4096;
        for (int32_t at = 0; at < sequences; at += kGridDim) {
            const int32_t count = sequences - at < kGridDim ? sequences - at : kGridDim;
            ctx.launch3d(read_kernel<D, B>, (unsigned)tiles, (unsigned)cache->heads, (unsigned)count, 256,
                         static_cast<uint16_t *>(k_out), static_cast<uint16_t *>(v_out), starts + at, rows,
                         Sequences{page_table + at * table_width, lengths + at, table_width}, pool_of(*cache));
        }
    });
    return ctx.status();
}

size_t equarx_cache_attention_workspace_bytes(int32_t heads, int32_t dim, int64_t q_rows, int32_t q_heads, int32_t sequences,
                                              int32_t max_queries, int64_t max_length)
{
    if (check_heads(heads, q_rows, q_heads, dim, sequences, max_queries, max_length) != EQUARX_OK || sequences == 0) return 0;
    return attention_workspace(plan_attention(heads, dim, q_heads, sequences, max_queries, max_length), dim, q_rows, q_heads);
}

size_t equarx_cache_attention_most_workspace_bytes(int32_t heads, int32_t dim, int64_t q_rows, int32_t q_heads, int32_t sequences,
                                                   int64_t max_length)
{
    if (check_heads(heads, q_rows, q_heads, dim, sequences, 1, max_length) != EQUARX_OK || sequences == 0 || q_rows == 0) return 0;
    return most_attention_workspace(heads, dim, q_rows, q_heads, sequences, max_length);
}

int equarx_cache_attention(const equarx_cache *cache, const void *q_bf16, int64_t q_rows, int32_t q_heads,
                           int64_t q_row_stride, int64_t q_head_stride, const int32_t *q_starts, const int32_t *page_table,
                           int64_t table_width, const int32_t *lengths, int32_t sequences, float scale, int32_t max_queries,
                           int64_t max_length, uint32_t flags, int32_t window, void *out_bf16, float *lse, void *workspace,
                           size_t workspace_bytes, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_cache(cache)) return st;
    if (int st = check_heads(cache->heads, q_rows, q_heads, cache->dim, sequences, max_queries, max_length)) return st;
    if (table_width < 1 || table_width > INT32_MAX || (flags & ~EQUARX_CAUSAL) != 0 || window < 0 ||
        (window > 0 && !(flags & EQUARX_CAUSAL)))
        return EQUARX_BAD_SHAPE;
    if (sequences == 0 || q_rows == 0) return EQUARX_OK;
    size_t q_bytes;
    if (int st = check_tokens(q_bf16, q_rows, q_heads, cache->dim, q_row_stride, q_head_stride, q_bytes)) return st;
    Aliasing mem;
    if (int st = check_sequences(page_table, table_width, lengths, sequences, mem)) return st;
    if (!q_starts || !out_bf16) return EQUARX_NULL_POINTER;
    if (misaligned(q_starts, sizeof(int32_t)) || misaligned(out_bf16, kAlign) || misaligned(lse, kAlign) ||
        misaligned(workspace, kWorkspaceAlign))
        return EQUARX_MISALIGNED;
    const AttentionPlan plan = plan_attention(cache->heads, cache->dim, q_heads, sequences, max_queries, max_length);
    const size_t need = attention_workspace(plan, cache->dim, q_rows, q_heads);
    if (need > 0 && !workspace) return EQUARX_NULL_POINTER;
    if (workspace_bytes < need) return EQUARX_WORKSPACE_TOO_SMALL;
    mem.reads(q_bf16, q_bytes);
    mem.reads(q_starts, ((size_t)sequences + 1) * sizeof(int32_t));
    list_cache(*cache, false, mem);
    mem.writes(out_bf16, (size_t)q_rows * q_heads * cache->dim * 2);
    mem.writes(lse, (size_t)q_rows * q_heads * sizeof(float));
    mem.writes(workspace, need);
    if (int st = mem.check()) return st;

    AttentionCall call{};
    call.q = static_cast<const uint16_t *>(q_bf16);
    call.q_row = q_row_stride;
    call.q_head = q_head_stride;
    call.q_starts = q_starts;
    call.out = static_cast<uint16_t *>(out_bf16);
    call.lse = lse;
    call.part = static_cast<float *>(workspace);
    call.q_rows = q_rows;
    call.q_heads = q_heads;
    call.group = q_heads / cache->heads;
    call.scale = scale * 1.44269504089f;
    call.causal = (flags & EQUARX_CAUSAL) != 0;
    call.window = window;
    call.chunk = plan.chunk;
    call.splits = plan.splits;
    call.sequences = sequences;
    with_geometry(cache->dim, cache->block, [&](auto dim, auto block) {
        constexpr int D = decltype(dim)::value, NB = D / decltype(block)::value;
        launch_attention<D, NB>(plan, call, {page_table, lengths, table_width}, pool_of(*cache), ctx);
    });
    return ctx.status();
}

}  // extern "C"
