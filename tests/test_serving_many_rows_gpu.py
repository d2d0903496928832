"""Cache calls of more rows or tokens than the threads of one launch can be counted in 32 bits."""
import pytest
import torch

from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_memory_back():
    yield
    torch.cuda.empty_cache()


# The joins of parts: four waves a row and head reach 2^32 threads at 2^24, one at 2^26.
@pytest.mark.parametrize("heads,sequences,queries,max_length,rows", ((1, 1, 1, 2000, 1 << 24), (2, 128, 1, 2000, 1 << 26),
                                                                     (1, 1, 2, 9 * 256, 1 << 24), (1, 1, 2, 512, 1 << 26)))
def test_rows_of_no_sequence(heads, sequences, queries, max_length, rows):
    """A few rows at the end of a long q are as they are in a call of their own; nothing else is written."""
    dim, group, page, length = 64, 32 if queries > 1 else 32 // heads, 16, 700
    q_heads = heads * group
    q_rows = rows // q_heads + 3
    pages = -(-length // page)
    cache = eq.alloc_cache(pages, heads, page, dim, 64)
    k, v = (torch.randn(length, heads, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (1, 2))
    eq.equarx_cache_write(cache, k, v, torch.arange(length, device="cuda"))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(sequences, 1)
    lengths = torch.full((sequences,), length, dtype=torch.int32, device="cuda")
    one = torch.randn(1, q_heads, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    new = sequences * queries
    answers = []
    for count in (new, q_rows):
        q = one.expand(count, q_heads, dim)
        first = count - new
        starts = (first + queries * torch.arange(sequences + 1)).to(torch.int32).cuda()
        out = torch.full((count, q_heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((count, q_heads), 9.0, device="cuda")
        work = eq.alloc_cache_attention_workspace(cache, count, q_heads, sequences, queries, max_length)
        eq.equarx_cache_attention(cache, q, starts, table, lengths, out, 0.125, queries, max_length, True, 0, lse, work)
        answers.append((out[first:].clone(), lse[first:].clone()))
        assert (out[:first] == 9).all() and (lse[:first] == 9).all()
        del out, lse, work
    (out, lse), (far_out, far_lse) = answers
    assert torch.equal(out, far_out) and torch.equal(lse, far_lse)
    assert (out != 9).any(dim=-1).all() and torch.isfinite(lse).all() and (lse != 9).all()


@pytest.mark.parametrize("dim", (64, 256))
def test_tokens_that_are_all_written(dim):
    """2^29 + 5 tokens, all of one key and value; a few of them have slots."""
    tokens, page = (1 << 29) + 5, 16
    cache, want = (eq.alloc_cache(2, 1, page, dim, 64) for _ in range(2))
    k, v = (torch.randn(1, 1, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (1, 2))
    slots = torch.full((tokens,), -1, dtype=torch.int64, device="cuda")
    places = [0, 1, (1 << 22) - 1, 1 << 22, (1 << 28) + 3, (1 << 29) - 1, 1 << 29, tokens - 1]
    for slot, t in enumerate(places):
        slots[t] = 3 * slot
    eq.equarx_cache_write(cache, k.expand(tokens, 1, dim), v.expand(tokens, 1, dim), slots)
    few = len(places)
    eq.equarx_cache_write(want, k.repeat(few, 1, 1), v.repeat(few, 1, 1), 3 * torch.arange(few, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(cache, want)) and cache.k_codes.any()
