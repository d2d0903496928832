"""Cache calls of many sequences, on both sides of where a launch goes by their number, and of enough tokens that a lane writes four."""
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq
from test_cache_gpu import GEOMETRIES, _same_cache

pytestmark = pytest.mark.gpu

# a sequence is one of these; some have no tokens, or no queries
LENGTHS = (1, 40, 0, 700, 17, 64, 3)


def _sequences(count, heads, dim, block, most_queries):
    """Caches of seven sequences, of which `count` sequences are copies; their queries."""
    page = 16
    pages = sum(-(-n // page) for n in LENGTHS)
    r = ref.CacheRef(pages, heads, page, dim, block)
    table = torch.full((len(LENGTHS), max(-(-n // page) for n in LENGTHS)), -1, dtype=torch.int32)
    g = torch.Generator().manual_seed(count)
    at = 0
    for b, n in enumerate(LENGTHS):
        c = -(-n // page)
        table[b, :c] = torch.arange(at, at + c)
        at += c
        if n:
            k, v = (torch.randn(n, heads, dim, generator=g).to(torch.bfloat16) for _ in "kv")
            r.write(k, v, r.slots_of(table[b].tolist(), n))
    kinds = torch.randint(0, len(LENGTHS), (count,), generator=g)
    news = torch.randint(0, most_queries + 1, (count,), generator=g)
    news[-1], kinds[-1] = 1, 3
    return r, table, kinds, news


def _check(count, heads, group, dim, block, max_queries, max_length, most_queries=1):
    r, table, kinds, news = _sequences(count, heads, dim, block, most_queries)
    starts = torch.cat((torch.zeros(1, dtype=torch.int64), news.cumsum(0))).to(torch.int32)
    rows, q_heads = int(news.sum()), heads * group
    q = torch.randn(rows, q_heads, dim, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    out, lse = torch.full((rows, q_heads, dim), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows, q_heads), 9.0, device="cuda")
    cache = r.device()
    lengths = torch.tensor(LENGTHS)[kinds]
    work = eq.alloc_cache_attention_workspace(cache, rows, q_heads, count, max_queries, max_length)
    work.fill_(0xFF)
    eq.equarx_cache_attention(cache, q.cuda(), starts.cuda(), table[kinds].cuda(), lengths.to(torch.int32).cuda(), out, dim ** -0.5, max_queries,
                              max_length, True, 0, lse, work)
    got, got_lse = out.double().cpu(), lse.double().cpu()
    # all queries that stand alike together, in 64 bits: query i of n at length - n + i
    sequence = torch.repeat_interleave(torch.arange(count), news)
    place = lengths[sequence] - news[sequence] + torch.arange(rows) - starts[:-1].long()[sequence]
    keys, values = r.values(0), r.values(1)
    for kind, n in enumerate(LENGTHS):
        for at in place[kinds[sequence] == kind].unique().tolist():
            here = ((kinds[sequence] == kind) & (place == at)).nonzero().flatten()
            if at < 0:
                assert (got[here] == 0).all() and torch.isneginf(got_lse[here]).all()
                continue
            slots = r.slots_of(table[kind].tolist(), n)[:at + 1]
            k, v = (x[slots].repeat_interleave(group, dim=1).transpose(0, 1) for x in (keys, values))      # [q_heads, tokens, dim]
            x = q[here].double().transpose(0, 1)
            s = dim ** -0.5 * (x @ k.transpose(1, 2))
            size = dim ** -0.5 * (x.abs() @ k.abs().transpose(1, 2)).amax(-1)
            want_lse = torch.logsumexp(s, -1)
            p = torch.exp(s - want_lse[..., None])
            want, mass = p @ v, p @ v.abs()
            e = (dim + 8) * 2.0 ** -23 * size + 2.0 ** -20 + (n + 64) * 2.0 ** -23
            bound = 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2.02 * e[..., None]) * mass
            assert ((got[here].transpose(0, 1) - want).abs() <= bound).all(), (kind, at)
            assert ((got_lse[here].T - want_lse).abs() <= 1.01 * e + 2.0 ** -21 * want_lse.abs()).all(), (kind, at)


# One of 256 threads counts one sequence, two, three or four; a last thread of theirs that ends with the sequences; above 1024 they are not
# shared out.
@pytest.mark.parametrize("count", (1, 255, 256, 257, 300, 511, 512, 513, 767, 768, 1000, 1023, 1024, 1025, 1100))
def test_single_tokens_of_many_sequences(count):
    _check(count, 2, 4, 64, 64, 1, 1024)


@pytest.mark.parametrize("count", (257, 512, 1024))
@pytest.mark.parametrize("dim,block", ((128, 64), (256, 128)))
def test_a_few_tokens_of_many_sequences(count, dim, block):
    _check(count, 1, 3, dim, block, 4, 1024, most_queries=4)


# A grid's second and third dimension reach to 65535.  One longest run gives the kernels for few rows, another that for many, whose
# sequences are in the third dimension or in the second.
@pytest.mark.parametrize("count", (65535, 65536, 65541, 131075))
@pytest.mark.parametrize("max_queries,max_length", ((1, 700), (40, 700), (400, 700)))
def test_more_sequences_than_a_grid_has(count, max_queries, max_length):
    _check(count, 1, 2, 64, 64, max_queries, max_length)


@pytest.mark.parametrize("count", (65535, 65541))
def test_reading_more_sequences_back_than_a_grid_has(count):
    r, table, kinds, _ = _sequences(count, 1, 64, 64, 1)
    kinds[kinds == 3] = 1                                       # the long one out: 40 tokens each
    lengths = torch.tensor(LENGTHS)[kinds]
    starts = lengths.cumsum(0) - lengths
    rows = int(lengths.sum())
    outs = [torch.full((rows, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    eq.equarx_cache_read(r.device(), table[kinds].cuda(), lengths.to(torch.int32).cuda(), starts.to(torch.int32).cuda(), *outs, 64)
    sequence = torch.repeat_interleave(torch.arange(count), lengths)
    token = torch.arange(rows) - starts[sequence]
    slots = table[kinds[sequence], token // 16].long() * 16 + token % 16
    for i, out in enumerate(outs):
        want = (r.codes[i].float() * r.scales[i].repeat_interleave(64, dim=-1)).to(torch.bfloat16)[slots]
        assert torch.equal(out.cpu(), want)


def _orders(tokens, slots):
    """Slots for tokens: in order from a group's first, from elsewhere, backwards, in fours, in sixteens, in no order, with gaps."""
    g = torch.Generator().manual_seed(tokens)
    t = torch.arange(tokens)
    by = lambda n: (torch.randperm(slots // n, generator=g)[:-(-tokens // n), None] * n + torch.arange(n)).flatten()[:tokens]
    gaps = 16 + t
    gaps[5::37], gaps[64:80], gaps[-1] = -1, slots + 3, slots
    return {"in order": t, "from the third": t + 3, "from a four": t + 4, "backwards": slots - 1 - t, "fours": by(4), "sixteens": by(16),
            "any": torch.randperm(slots, generator=g)[:tokens], "gaps": gaps}


@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("order", sorted(_orders(100, 200)))
def test_four_tokens_a_lane(dim, block, order):
    """Enough tokens for a workgroup on every CU: the same codes and scales as ever, whatever the order of the slots."""
    heads, page = 8, 48
    tokens = 256 // heads * (256 // (dim // 8) * 4) + 21
    pages = -(-tokens // page) + 2
    slots = _orders(tokens, pages * page)[order]
    r, cache = ref.CacheRef(pages, heads, page, dim, block), eq.alloc_cache(pages, heads, page, dim, block)
    x = torch.randn(tokens, (2 * heads + 1) * dim, generator=torch.Generator().manual_seed(dim)).to(torch.bfloat16)
    x[30, dim + 5], x[77, -3], x[100, dim:dim + block] = float("nan"), float("inf"), 0
    k, v = (x[:, (1 + i * heads) * dim:][:, :heads * dim].view(tokens, heads, dim) for i in (0, 1))
    dev = x.cuda()
    dk, dv = (dev[:, (1 + i * heads) * dim:][:, :heads * dim].view(tokens, heads, dim) for i in (0, 1))
    eq.equarx_cache_write(cache, dk, dv, slots.cuda())
    r.write(k, v, slots)
    _same_cache(cache, r)
