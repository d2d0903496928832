"""Page tables whose rows stay where they were asked for, on the GPU against a plain statement of what they hold."""
import pytest
import torch

import test_pages_gpu as compact
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def _model_extend(m, counts, rows, tags, pages):
    """On a test_pages_gpu.Model: starts, granted, what rows are told, seen."""
    at, wanted_rows, wanted_pages = len(m.free), 0, 0
    starts, granted, told, seen = [0], [], [], []
    for b, row in enumerate(m.table):
        n, asked = m.length(b), max(counts[b], 0)
        wanted_rows += asked
        fits = n + asked <= len(row) * m.page and n + asked <= 2 ** 31 - 1 and wanted_rows <= rows
        need = m.up(n + asked) - m.up(n) if fits else 0
        wanted_pages += need
        want = asked if fits and (need == 0 or wanted_pages <= at) else 0
        for i in range(need if want else 0):
            row[m.up(n) + i] = m.free.pop()
        m.lengths[b] = n + want
        granted.append(want)
        seen.append(0 if asked and not want else n + want)
        starts.append(min(wanted_rows, rows))
        for t in range(starts[-1] - starts[-2]):
            p = row[(n + t) // m.page] if want else -1
            told.append((p * m.page + (n + t) % m.page if 0 <= p < pages else -1, n + t if want else -1, tags[b] if want else -1))
    return starts, granted, told + [(-1, -1, -1)] * (rows - len(told)), seen


def _extend(pages, model, counts, rows):
    sequences, total = len(counts), pages.free.numel()
    ints = lambda n, dtype=torch.int32: torch.full((n,), 12345, dtype=dtype, device="cuda")
    starts, slots, granted, positions, row_tags, seen = ints(sequences + 1), ints(rows, torch.int64), ints(sequences), ints(rows), ints(rows), ints(sequences)
    tags = [3 * b - 1 for b in range(sequences)]
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    eq.equarx_pages_extend(pages, model.page, on(counts), starts, slots, granted, positions, on(tags), row_tags, seen)
    want_starts, want_granted, told, want_seen = _model_extend(model, counts, rows, tags, total)
    assert granted.tolist() == want_granted and starts.tolist() == want_starts and seen.tolist() == want_seen
    assert slots.tolist() == [t[0] for t in told]
    assert positions.tolist() == [t[1] for t in told]
    assert row_tags.tolist() == [t[2] for t in told]
    compact._check(pages, model, total)
    return want_granted


@pytest.mark.parametrize("sequences,width,total,page,seed", ((1, 1, 1, 1, 0), (1, 9, 20, 16, 1), (5, 7, 30, 16, 2), (17, 3, 40, 64, 3), (64, 33, 1500, 16, 4),
                                                             (70, 200, 9000, 17, 5), (1030, 5, 3000, 3, 6), (2100, 2, 3000, 128, 7)))
def test_sequences_come_and_go(sequences, width, total, page, seed):
    g = torch.Generator().manual_seed(seed)
    pages, model = compact._new(sequences, width, total, page)
    random = lambda hi: torch.randint(0, hi + 1, (sequences,), generator=g).tolist()
    most = width * page
    for step in range(8):
        kind = step % 4
        counts = random(most // 2) if kind == 0 else [1] * sequences if kind == 1 else random(most + 1) if kind == 2 else [c - 1 for c in random(3)]
        wanted = sum(max(c, 0) for c in counts)
        rows = [wanted + 3, wanted, wanted // 2, wanted + 100][(step + seed + step // 4) % 4]
        if rows > 60000:
            counts = [c % 7 for c in counts]
            rows = sum(counts) + 5
        _extend(pages, model, counts, rows)
        compact._trim(pages, model, [n if step % 2 else max(n - 5, 0) for n in random(most)] if step != 5 else [0] * sequences)


def test_rows_of_what_gets_nothing_stay_empty():
    pages, model = compact._new(4, 2, 5, 16)
    assert _extend(pages, model, [33, 32, 20, 17], 110) == [0, 32, 20, 0]               # the table; the stack
    assert _extend(pages, model, [33, 32, 20, 17], 100) == [0, 0, 0, 0]
    assert _extend(pages, model, [0, 1, 12, 16], 29) == [0, 0, 12, 16]                  # no page is needed, or the last one
    compact._trim(pages, model, [0, 5, 32, 0])
    assert _extend(pages, model, [10, 10, -3, 10], 19) == [10, 0, 0, 0]                 # rows: the second's end beyond the last
    assert _extend(pages, model, [0, 0, 0, 0], 7) == [0, 0, 0, 0]


@pytest.mark.parametrize("rows", (50, 5000))
def test_counts_past_all_rows(rows):
    """Sums of what is wanted that pass 32 bits."""
    pages, model = compact._new(1500, 2, 3000, 16)
    for big in (2 ** 31 - 1, 2 ** 30, 2 ** 30 + 1):
        counts = [1, 0, 3] * 500
        for b in (7, 8, 9, 700, 1100, 1101, 1102):
            counts[b] = big
        granted = _extend(pages, model, counts, rows)
        assert granted[:7] == counts[:7] and not any(granted[7:])
        _extend(pages, model, [0] * 1499 + [big], rows)


def test_rows_of_two_launches():
    pages, model = compact._new(30, 300, 700, 16)
    assert _extend(pages, model, [4000, 0, 1, 4801, 700] + [129] * 25, 40000)[3] == 0
    _extend(pages, model, [1] * 30, 5000)
    _extend(pages, model, [129] * 30, 4500)
    pages, model = compact._new(1200, 40, 2000, 16)
    _extend(pages, model, [7] * 1199 + [600], 9000)
    _extend(pages, model, [14] * 1199 + [30], 17000)


def test_all_that_is_given_is_as_without():
    """Where all get what they want, the rows are those of the tokens."""
    for seen in (False, True):
        pages, model = compact._new(9, 10, 90, 16)
        extend = _extend if seen else compact._extend
        extend(pages, model, [5, 0, 17, 160, 1, 1, 0, 33, 16], 240)
        if not seen:
            want = [t.clone() for t in pages]
    assert all(torch.equal(a, b) for a, b in zip(want, pages))


def test_a_captured_step_goes_on_by_itself():
    """The stack runs out between replays, and is filled again."""
    pages, model = compact._new(4, 9, 9, 16)
    _extend(pages, model, [14, 30, 1, 60], 105)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    counts, keep, tags = on([1, 1, 1, 2]), on([1 << 20] * 4), on([5, 6, 7, 8])
    starts, slots, row_tags, positions, granted, seen = on([0] * 5), torch.zeros(8, dtype=torch.int64, device="cuda"), on([0] * 8), on([0] * 8), on([0] * 4), on([0] * 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eq.equarx_pages_trim(pages, 16, keep)
        eq.equarx_pages_extend(pages, 16, counts, starts, slots, granted, positions, tags, row_tags, seen)
    refused = 0
    for step in range(9):
        keep[0] = 3 if step == 6 else 1 << 20
        graph.replay()
        torch.cuda.synchronize()
        model.trim(keep.tolist(), 9)
        want_starts, want_granted, told, want_seen = _model_extend(model, counts.tolist(), 8, [5, 6, 7, 8], 9)
        assert starts.tolist() == want_starts and granted.tolist() == want_granted and seen.tolist() == want_seen
        assert list(zip(slots.tolist(), positions.tolist(), row_tags.tolist())) == told
        compact._check(pages, model, 9)
        refused += want_granted.count(0)
    assert refused > 3 and want_granted[0] == 1
