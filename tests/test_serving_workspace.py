"""The workspace of attention calls of several sizes, on the host: what the library says is enough for all, against what each needs."""
import pytest

from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build

# heads, query heads, dim, rows, sequences, tokens
LIMITS = [(8, 32, 128, 512, 64, 512), (4, 160, 128, 96, 12, 4096), (2, 8, 64, 53, 3, 40), (1, 1, 128, 300, 7, 131072), (1, 300, 64, 24, 5, 9000),
          (16, 16, 256, 130, 9, 2000), (2, 34, 256, 64, 4, 70000), (600, 600, 64, 40, 4, 3000), (8, 64, 128, 1, 1, 4096), (1, 16, 64, 1, 1, 600),
          (3, 60, 128, 20, 2000, 100000)]


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return eq.load()


@pytest.mark.parametrize("heads,q_heads,dim,rows,sequences,longest", LIMITS)
def test_what_is_enough_for_all_calls_is(lib, heads, q_heads, dim, rows, sequences, longest):
    """Every number of rows and sequences up to the limits, every longest run that the rows of a sequence allow and some that are
    longer than any; and not more than twice what one of them needs."""
    most = lib.equarx_cache_attention_most_workspace_bytes(heads, dim, rows, q_heads, sequences, longest)
    largest = 0
    for s in sorted({*range(1, min(sequences, 64) + 1), sequences, max(sequences - 1, 1), min(sequences, 1024), min(sequences, 1025)}):
        for r in sorted({*range(1, min(rows, 40) + 1), *range(1, rows + 1, 7), rows}):
            for queries in {*range(-(-r // s), min(r, 40) + 1), *range(-(-r // s), r + 1, 5), r, r + 1, 2 * r, 40 * r, 5000}:
                if queries * s < r:
                    continue
                for length in (longest, longest // 2 + 1):
                    largest = max(largest, lib.equarx_cache_attention_workspace_bytes(heads, dim, r, q_heads, s, queries, length))
    assert largest <= most <= 2 * largest


def test_what_holds_nothing_or_is_refused_needs_nothing(lib):
    most = lib.equarx_cache_attention_most_workspace_bytes
    assert most(2, 128, 20, 8, 4, 5000) > 0
    for changed in ((2, 96, 20, 8, 4, 5000), (2, 128, -1, 8, 4, 5000), (2, 128, 20, 7, 4, 5000), (2, 128, 20, 8, -1, 5000), (2, 128, 20, 8, 4, 0),
                    (2, 128, 0, 8, 4, 5000), (2, 128, 20, 8, 0, 5000), (0, 128, 20, 8, 4, 5000)):
        assert most(*changed) == 0, changed


def test_a_product_of_fewer_rows_needs_no_more(lib):
    """What a layer's workspace takes for granted of the 4-bit products."""
    size = lib.equarx_mx4_workspace_bytes
    for n, k in ((96, 300), (5376, 4096), (1, 40), (64, 1 << 20)):
        needs = [size(m, n, k) for m in range(1, 300)]
        assert needs == sorted(needs)


def test_the_binding_asks_for_either(lib):
    cache = eq.alloc_cache(2, 8, 16, 128, 64, device="meta")
    sizes = [eq.alloc_cache_attention_workspace(cache, 512, 32, 64, q, 512, device="meta").numel() for q in (512, None)]
    assert sizes[0] == 256 and sizes[1] == lib.equarx_cache_attention_most_workspace_bytes(8, 128, 512, 32, 64, 512)
