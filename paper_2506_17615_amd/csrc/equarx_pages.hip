// Host side of the page tables' calls: argument validation and launch.
#include "equarx.h"

#include "equarx_launch.hpp"
#include "equarx_pages.hpp"

namespace {

using namespace equarx;
using namespace equarx::host;
using namespace equarx::pages;

constexpr int64_t kMostElements = (int64_t)1 << 40, kMostRows = (int64_t)1 << 30, kMostPages = (int64_t)1 << 30;
constexpr int32_t kMostSequences = 1 << 20, kMostWidth = 1 << 20;

int check_pages(const equarx_pages *p)
{
    if (!p) return EQUARX_NULL_POINTER;
    if (p->sequences < 0 || p->sequences > kMostSequences || p->width < 1 || p->width > kMostWidth || p->pages < 1 ||
        p->pages > kMostPages || p->page < 1 || p->page > 65536)
        return EQUARX_BAD_SHAPE;
    if (p->pages > kMostElements / p->page) return EQUARX_BAD_SHAPE;
    if (p->sequences == 0) return EQUARX_OK;
    if (p->width > kMostElements / p->sequences) return EQUARX_BAD_SHAPE;
    if (!p->table || !p->lengths || !p->free || !p->free_count) return EQUARX_NULL_POINTER;
    if (misaligned(p->table, 4) || misaligned(p->lengths, 4) || misaligned(p->free, 4) || misaligned(p->free_count, 4)) return EQUARX_MISALIGNED;
    return EQUARX_OK;
}

Pool pool_of(const equarx_pages &p)
{
    const int64_t room = p.width * p.page;
    return {p.table, p.lengths, p.free, p.free_count, p.seen, p.width, (int32_t)p.pages, p.sequences, (int32_t)(room < INT32_MAX ? room : INT32_MAX),
            Divisor((uint32_t)p.page)};
}

void list_pages(const equarx_pages &p, Aliasing &mem)
{
    mem.writes(p.table, (size_t)(p.width * p.sequences) * 4);
    mem.writes(p.lengths, (size_t)p.sequences * 4);
    mem.writes(p.free, (size_t)p.pages * 4);
    mem.writes(p.free_count, 4);
}

// Rows that the workgroup which hands out the pages tells as well; more get a launch of their own, which is 2.3 us by itself.  Measured on MI355X, us of
// trim and extend, in two launches -> in three, of 8 and of 64 sequences: 1000 rows 7.2, 7.5 -> 9.6, 10.2; 2000 7.9, 8.8 -> 9.7; 4100 9.4, 10.2 -> 9.8, 9.6;
// 8200 11.8, 13.5 -> 9.8, 9.6.
constexpr int64_t kToldAtOnce = 4096;

}  // namespace

extern "C" {

int equarx_pages_trim(const equarx_pages *pages, const int32_t *keep, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_pages(pages)) return st;
    if (pages->sequences == 0) return EQUARX_OK;
    if (!keep) return EQUARX_NULL_POINTER;
    if (misaligned(keep, 4)) return EQUARX_MISALIGNED;
    Aliasing mem;
    list_pages(*pages, mem);
    mem.reads(keep, (size_t)pages->sequences * 4);
    if (int st = mem.check()) return st;
    ctx.launch(trim_kernel, 1, kTeam, pool_of(*pages), keep);
    return ctx.status();
}

int equarx_pages_extend(const equarx_pages *pages, const int32_t *counts, int32_t *q_starts, int64_t *slots, int32_t *granted,
                        int32_t *positions, const int32_t *tags, int32_t *row_tags, int64_t rows, void *stream)
{
    LaunchCtx ctx(stream);
    if (int st = check_pages(pages)) return st;
    if (rows < 0 || rows > kMostRows) return EQUARX_BAD_SHAPE;
    if (pages->sequences == 0 && rows == 0 && !q_starts) return EQUARX_OK;
    if (!q_starts || (pages->sequences > 0 && !counts) || (rows > 0 && !slots)) return EQUARX_NULL_POINTER;
    if (rows > 0 && pages->sequences > 0 && !tags != !row_tags) return EQUARX_NULL_POINTER;
    if (misaligned(pages->seen, 4) || misaligned(counts, 4) || misaligned(q_starts, 4) || misaligned(slots, 8) || misaligned(granted, 4) || misaligned(positions, 4) ||
        misaligned(tags, 4) || misaligned(row_tags, 4))
        return EQUARX_MISALIGNED;
    Aliasing mem;
    const size_t sequences = (size_t)pages->sequences;
    if (sequences > 0) list_pages(*pages, mem);
    mem.reads(counts, sequences * 4);
    mem.reads(tags, sequences * 4);
    mem.writes(q_starts, (sequences + 1) * 4);
    mem.writes(granted, sequences * 4);
    mem.writes(pages->seen, sequences * 4);
    mem.writes(slots, (size_t)rows * 8);
    mem.writes(positions, (size_t)rows * 4);
    mem.writes(row_tags, (size_t)rows * 4);
    if (int st = mem.check()) return st;
    const Pool p = pool_of(*pages);
    const Rows to{slots, positions, row_tags, tags, (int32_t)rows};
    const bool at_once = rows <= kToldAtOnce;
    ctx.launch(extend_kernel, 1, kTeam, p, counts, q_starts, granted, to, at_once);
    if (!at_once) ctx.launch(tell_kernel, (unsigned)((rows + 255) / 256), 256, p, static_cast<const int32_t *>(q_starts), to);
    return ctx.status();
}

}  // extern "C"
