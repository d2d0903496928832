"""Page tables on the GPU against a plain statement of what they hold: whole numbers, which have one right answer."""
import ctypes

import pytest
import torch

from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


class Model:
    """Lists of Python integers."""

    def __init__(self, table, lengths, free, page):
        self.table, self.lengths, self.free, self.page = [list(r) for r in table], list(lengths), list(free), page

    def up(self, n):
        return -(-n // self.page)

    def length(self, b):
        return min(max(self.lengths[b], 0), len(self.table[b]) * self.page)

    def trim(self, keep, pages):
        for b, row in enumerate(self.table):
            n = self.length(b)
            kept = min(max(keep[b], 0), n)
            for i in range(self.up(kept), self.up(n)):
                if 0 <= row[i] < pages and len(self.free) < pages:
                    self.free.append(row[i])
                row[i] = -1
            self.lengths[b] = kept

    def extend(self, counts, rows, tags, pages):
        starts, granted, told = [0], [], []
        wanted_rows = wanted_pages = 0
        for b, row in enumerate(self.table):
            n, want = self.length(b), max(counts[b], 0)
            if n + want > len(row) * self.page or n + want > 2 ** 31 - 1:
                want = 0
            wanted_rows += want
            if wanted_rows > rows:
                want = 0
            need = self.up(n + want) - self.up(n)
            wanted_pages += need
            granted.append((b, n, want, need, wanted_pages))
        at = list(self.free)
        for b, n, want, need, upto in granted:
            row = self.table[b]
            if need and upto > len(at):
                want = need = 0
            for i in range(need):
                row[self.up(n) + i] = self.free.pop()
            self.lengths[b] = n + want
            starts.append(starts[-1] + want)
            for t in range(n, n + want):
                p = row[t // self.page]
                told.append((p * self.page + t % self.page if 0 <= p < pages else -1, t, tags[b]))
        told += [(-1, -1, -1)] * (rows - len(told))
        return starts, [s - r for r, s in zip(starts, starts[1:])], told


def _check(pages, model, count):
    assert pages.table.tolist() == model.table
    assert pages.lengths.tolist() == model.lengths
    n = int(pages.free_count)
    assert n == len(model.free) and pages.free[:n].tolist() == model.free


def _extend(pages, model, counts, rows, tags=None):
    sequences, total = len(counts), pages.free.numel()
    ints = lambda n, dtype=torch.int32: torch.full((n,), 12345, dtype=dtype, device="cuda")
    starts, slots, granted, positions, row_tags = ints(sequences + 1), ints(rows, torch.int64), ints(sequences), ints(rows), ints(rows)
    tags = [3 * b - 1 for b in range(sequences)] if tags is None else tags
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    eq.equarx_pages_extend(pages, model.page, on(counts), starts, slots, granted, positions, on(tags), row_tags)
    want_starts, want_granted, told = model.extend(counts, rows, tags, total)
    assert starts.tolist() == want_starts and granted.tolist() == want_granted
    assert slots.tolist() == [t[0] for t in told]
    assert positions.tolist() == [t[1] for t in told]
    assert row_tags.tolist() == [t[2] for t in told]
    _check(pages, model, total)
    return want_granted


def _trim(pages, model, keep):
    eq.equarx_pages_trim(pages, model.page, torch.tensor(keep, dtype=torch.int32, device="cuda"))
    model.trim(keep, pages.free.numel())
    _check(pages, model, pages.free.numel())


def _new(sequences, width, total, page):
    pages = eq.alloc_pages(sequences, width, total)
    return pages, Model(pages.table.tolist(), pages.lengths.tolist(), pages.free.tolist(), page)


@pytest.mark.parametrize("sequences,width,total,page,seed", ((1, 1, 1, 1, 0), (1, 9, 20, 16, 1), (5, 7, 30, 16, 2), (17, 3, 40, 64, 3),
                                                             (64, 33, 1500, 16, 4), (70, 200, 9000, 17, 5), (1030, 5, 3000, 3, 6),
                                                             (2100, 2, 5000, 128, 7)))
def test_sequences_come_and_go(sequences, width, total, page, seed):
    """Steps of random counts and keeps, some of them more than table, rows or stack hold."""
    g = torch.Generator().manual_seed(seed)
    pages, model = _new(sequences, width, total, page)
    random = lambda hi: torch.randint(0, hi + 1, (sequences,), generator=g).tolist()
    most = width * page
    for step in range(7):
        kind = step % 4
        counts = random(most // 2) if kind == 0 else [1] * sequences if kind == 1 else random(most + 1) if kind == 2 else random(2)
        wanted = sum(counts)
        rows = [wanted + 3, wanted, wanted // 2, wanted + 100][(step + seed) % 4]
        if rows > 60000:
            counts = [c % 7 for c in counts]
            rows = sum(counts) + 5
        _extend(pages, model, counts, rows)
        _trim(pages, model, [n if step % 2 else max(n - 5, 0) for n in random(most)] if step != 5 else [0] * sequences)


def test_every_token_has_a_slot_of_its_own():
    pages, model = _new(40, 30, 700, 16)
    for counts in ([16] * 40, [1] * 40, [100] * 40, [37] * 40):
        _extend(pages, model, counts, sum(counts))
    held = []
    for b, n in enumerate(pages.lengths.tolist()):
        held += pages.table[b, :-(-n // 16)].tolist()
    free = pages.free[:int(pages.free_count)].tolist()
    assert sorted(held + free) == list(range(700))


def test_rows_of_two_launches():
    """More rows than are told by the workgroup that hands out the pages."""
    pages, model = _new(30, 300, 9000, 16)
    _extend(pages, model, [4000, 0, 1, 4800, 700] + [129] * 25, 40000)
    _extend(pages, model, [1] * 30, 5000)


def test_what_has_no_room_gets_nothing():
    pages, model = _new(4, 2, 5, 16)
    assert _extend(pages, model, [33, 32, 20, 17], 100) == [0, 32, 20, 0]               # the table; the stack
    assert _extend(pages, model, [0, 1, 12, 16], 100) == [0, 0, 12, 16]                 # no page is needed, or the last one
    assert _extend(pages, model, [1, 0, 0, 0], 100) == [0, 0, 0, 0]
    _trim(pages, model, [0, 5, 32, 0])
    assert _extend(pages, model, [10, 10, 0, 10], 19) == [10, 0, 0, 0]                  # rows: nor anything after the first too many
    assert _extend(pages, model, [-5, 3, 0, 0], 3) == [0, 3, 0, 0]


def test_no_rows_and_no_counts():
    pages, model = _new(3, 4, 8, 16)
    _extend(pages, model, [0, 0, 0], 7)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    starts = on([9, 9, 9, 9])
    eq.equarx_pages_extend(pages, 16, on([1, 0, 2]), starts, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert starts.tolist() == [0, 0, 0, 0] and pages.lengths.tolist() == [0, 0, 0]


@pytest.mark.parametrize("rows", (1, 300, 5000))
def test_no_sequences(rows):
    """Every row is told that it is nobody's; there need be no pages, and what there is stays."""
    pages, ints = eq.alloc_pages(0, 4, 8), lambda n, dtype=torch.int32: torch.full((n,), 12345, dtype=dtype, device="cuda")
    pages.free_count.fill_(77)
    starts, slots, positions = ints(1), ints(rows, torch.int64), ints(rows)
    for own in (eq._CPages(None, None, pages.free.data_ptr(), pages.free_count.data_ptr(), 4, 8, 0, 16), eq._CPages(None, None, None, None, 4, 8, 0, 16)):
        for t in (starts, slots, positions):
            t.fill_(12345)
        assert eq.load().equarx_pages_extend(ctypes.byref(own), None, starts.data_ptr(), slots.data_ptr(), None, positions.data_ptr(), None, None, rows,
                                             torch.cuda.current_stream().cuda_stream) == 0
        assert starts.tolist() == [0] and (slots == -1).all() and (positions == -1).all() and int(pages.free_count) == 77
    slots.fill_(5)
    eq.equarx_pages_extend(pages, 16, ints(0), starts, slots)
    assert starts.tolist() == [0] and (slots == -1).all() and int(pages.free_count) == 77


def test_values_out_of_range():
    """Lengths past the table, below zero, entries that are no page, a stack that says it holds more than it can."""
    pages, model = _new(4, 3, 9, 16)
    _extend(pages, model, [40, 20, 16, 3], 100)
    pages.lengths.copy_(torch.tensor([1000, -7, 16, 3]))
    pages.table[0, 1], pages.table[2, 0] = 1 << 20, -9
    model.lengths, model.table = [1000, -7, 16, 3], pages.table.tolist()
    _trim(pages, model, [0, 0, 3, 100])
    _extend(pages, model, [1, 1, 1, 1], 9)
    pages.free_count.fill_(1 << 30)
    starts, slots = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(50, dtype=torch.int64, device="cuda")
    eq.equarx_pages_extend(pages, 16, torch.tensor([9] * 4, dtype=torch.int32, device="cuda"), starts, slots)
    assert 0 <= int(pages.free_count) <= 9 and (slots >= -1).all() and (slots < 9 * 16).all()
    pages.free_count.fill_(-5)
    eq.equarx_pages_trim(pages, 16, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert 0 <= int(pages.free_count) <= 9


def test_a_long_context():
    pages, model = _new(2, 70000, 140000, 16)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    starts, slots = on([0, 0, 0]), torch.zeros(2 * 1048576 + 1, dtype=torch.int64, device="cuda")
    eq.equarx_pages_extend(pages, 16, on([1048576, 1048576]), starts, slots)
    assert starts.tolist() == [0, 1048576, 2097152] and int(pages.free_count) == 140000 - 131072 and slots[-1] == -1
    t = torch.arange(1048576, device="cuda")
    for b in range(2):
        want = pages.table[b, t // 16].long() * 16 + t % 16
        assert torch.equal(slots[b * 1048576:(b + 1) * 1048576], want)
    assert slots[:-1].unique().numel() == 2097152
    eq.equarx_pages_trim(pages, 16, on([17, 0]))
    assert int(pages.free_count) == 139998 and pages.free[:139998].unique().numel() == 139998
    assert (pages.table[0, 2:] == -1).all() and (pages.table[1] == -1).all()


def test_a_captured_step_goes_on_by_itself():
    """Decode steps of a graph, eager calls between its replays: sequence 1 ends after three, sequence 3 has two tokens a step."""
    pages, model = _new(4, 9, 30, 16)
    _extend(pages, model, [14, 30, 1, 60], 200)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    counts, keep, tags = on([1, 1, 1, 2]), on([1 << 20] * 4), on([5, 6, 7, 8])
    starts, slots, row_tags, positions, granted = on([0] * 5), torch.zeros(8, dtype=torch.int64, device="cuda"), on([0] * 8), on([0] * 8), on([0] * 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eq.equarx_pages_trim(pages, 16, keep)
        eq.equarx_pages_extend(pages, 16, counts, starts, slots, granted, positions, tags, row_tags)
    for step in range(6):
        if step == 3:
            keep[1], counts[1] = 0, 0
        graph.replay()
        torch.cuda.synchronize()
        model.trim(keep.tolist(), 30)
        want_starts, want_granted, told = model.extend(counts.tolist(), 8, [5, 6, 7, 8], 30)
        assert starts.tolist() == want_starts and granted.tolist() == want_granted
        assert list(zip(slots.tolist(), positions.tolist(), row_tags.tolist())) == told
        _check(pages, model, 30)
        if step == 4:
            _extend(pages, model, [0, 31, 0, 0], 40)                 # a new request between two replays
            keep[1], counts[1] = 1 << 20, 1


def test_another_stream():
    pages, model = _new(6, 4, 20, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _extend(pages, model, [20, 1, 0, 16, 17, 2], 60)
        _trim(pages, model, [3, 0, 0, 16, 16, 1])
