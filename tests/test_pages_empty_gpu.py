"""A step of no sequences and no rows tells that it has none."""
import ctypes

import pytest
import torch

from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def test_no_sequences_and_no_rows():
    pages, ints = eq.alloc_pages(0, 4, 8), lambda n: torch.full((n,), 12345, dtype=torch.int32, device="cuda")
    starts, slots = ints(1), torch.empty(0, dtype=torch.int64, device="cuda")
    eq.equarx_pages_extend(pages, 16, ints(0), starts, slots)
    assert starts.tolist() == [0] and int(pages.free_count) == 8
    starts = ints(1)
    eq.equarx_pages_extend(pages, 16, ints(0), starts, slots, seen=ints(0))
    assert starts.tolist() == [0]
    starts = ints(1)
    none = eq._CPages(None, None, None, None, 4, 8, 0, 16)
    stream = torch.cuda.current_stream().cuda_stream
    assert eq.load().equarx_pages_extend(ctypes.byref(none), None, starts.data_ptr(), None, None, None, None, None, 0, stream) == 0
    assert starts.tolist() == [0]
