"""The int8 key/value cache and its attention on the GPU against plain statements in 64 bits.

Writing has one right answer, reading back too.  Attention's bound, per output element: half a bf16 unit of the result (2^-8);
the products p * v-scale rounded to bf16 (2^-8 of sum p |v|); an error e of the scores, which moves p by that share, with
e = (dim + 8) 2^-23 of the largest sum |q k| |scale| for the fp32 dot product plus 2^-20 for the exponential and its argument,
and (tokens + 64) 2^-23 for the sums."""
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu
GEOMETRIES = ((64, 64), (128, 64), (128, 128), (256, 64), (256, 128), (256, 256))


def _bf16(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _same_cache(cache, r):
    want = r.device("cpu")
    finite = [torch.isfinite(s.cpu()) for s in (want.k_scales, want.v_scales)]
    for got, ok, alive in ((cache.k_scales, want.k_scales, finite[0]), (cache.v_scales, want.v_scales, finite[1])):
        assert torch.equal(torch.isnan(got.cpu()), ~alive) and torch.equal(got.cpu()[alive], ok[alive])
    per = r.block
    k_alive = finite[0].permute(0, 1, 3, 2).repeat_interleave(per, dim=-1)
    v_alive = finite[1].view(*finite[1].shape[:3], -1, 16).permute(0, 1, 3, 2, 4).repeat_interleave(per, dim=3)
    assert torch.equal(cache.k_codes.cpu()[k_alive], want.k_codes[k_alive])
    assert torch.equal(cache.v_codes.cpu()[v_alive], want.v_codes[v_alive])


@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("page,tokens,heads", ((16, 1, 3), (48, 67, 2), (64, 130, 1)))
def test_write(dim, block, page, tokens, heads):
    pages = -(-tokens // page) + 2
    r = ref.CacheRef(pages, heads, page, dim, block)
    cache = eq.alloc_cache(pages, heads, page, dim, block)
    qkv = _bf16(tokens + dim, tokens, (2 * heads + 1) * dim)                # keys and values inside a fused projection
    qkv[0, dim:dim + block] = 0
    qkv[-1, (1 + heads) * dim:(1 + heads) * dim + block] = 2.0 ** -130      # below the smallest scale
    k, v = (qkv[:, (1 + i * heads) * dim:(1 + (i + 1) * heads) * dim].view(tokens, heads, dim) for i in (0, 1))
    g = torch.Generator().manual_seed(tokens)
    start = 5 if tokens > 1 else 0
    for slots in (torch.arange(start, start + tokens), torch.randperm(pages * page, generator=g)[:tokens]):
        slots = slots.clone()
        if tokens > 20:
            slots[7], slots[11] = -1, pages * page                          # skipped
        dev = qkv.cuda()
        dk, dv = (dev[:, (1 + i * heads) * dim:(1 + (i + 1) * heads) * dim].view(tokens, heads, dim) for i in (0, 1))
        eq.equarx_cache_write(cache, dk, dv, slots.cuda())
        r.write(k, v, slots)
        _same_cache(cache, r)


def test_codes_and_scales_are_those_of_the_wire():
    """A token's key is quantized as equarx_quantize would quantize it."""
    heads, dim, block = 4, 128, 64
    x = _bf16(1, 16, heads, dim).cuda()
    cache = eq.alloc_cache(1, heads, 16, dim, block)
    eq.equarx_cache_write(cache, x, x, torch.arange(16, device="cuda"))
    codes = torch.empty(x.numel(), dtype=torch.int8, device="cuda")
    scales = torch.empty(x.numel() // block, dtype=torch.float32, device="cuda")
    eq.equarx_quantize(x.reshape(-1), block, codes, scales)
    assert torch.equal(cache.k_codes[0].permute(1, 0, 2).reshape(-1), codes)
    assert torch.equal(cache.k_scales[0].permute(2, 0, 1).reshape(-1), scales)


@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_a_block_that_is_not_finite_gets_a_nan_scale(bad):
    r, cache = ref.CacheRef(2, 2, 16, 128, 64), eq.alloc_cache(2, 2, 16, 128, 64)
    k, v = _bf16(2, 20, 2, 128), _bf16(3, 20, 2, 128)
    k[4, 1, 70], v[9, 0, 3] = bad, -bad
    r.write(k, v, torch.arange(20))
    eq.equarx_cache_write(cache, k.cuda(), v.cuda(), torch.arange(20, device="cuda"))
    _same_cache(cache, r)


def _filled(seed, lengths, page, heads, dim, block, spare=1):
    """A cache of sequences in scattered pages, its table and the reference."""
    counts = [-(-n // page) for n in lengths]
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(counts + [1])
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    r = ref.CacheRef(pages, heads, page, dim, block)
    for b, c in enumerate(counts):
        table[b, :c] = torch.tensor([order.pop() for _ in range(c)], dtype=torch.int32)
        n = lengths[b]
        if n:
            r.write(_bf16(seed + b, n, heads, dim), _bf16(seed + 100 + b, n, heads, dim), r.slots_of(table[b].tolist(), n))
    return r, table


@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("page", (16, 48, 64))
def test_read_back(dim, block, page):
    lengths = [0, 1, 17, 130, 64]
    r, table = _filled(7, lengths, page, 3, dim, block)
    table[3, 1] = r.pages                                                   # a page that does not exist: zeros
    rows = sum(lengths) + 4
    starts = torch.tensor([0, 2, 3, 20, rows - 30], dtype=torch.int32)      # the last one runs over the end
    outs = [torch.full((rows, 3, dim), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    eq.equarx_cache_read(r.device(), table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts.cuda(), *outs)
    for i, out in enumerate(outs):
        want = torch.full((rows, 3, dim), 9.0, dtype=torch.bfloat16)
        exact = (r.codes[i].float() * r.scales[i].repeat_interleave(block, dim=-1)).to(torch.bfloat16)
        for b, n in enumerate(lengths):
            slots = r.slots_of(table[b].tolist(), n)
            got = torch.where((slots >= 0)[:, None, None], exact[slots.clamp(min=0)], 0.0)
            at = int(starts[b])
            want[at:min(at + n, rows)] = got[:max(0, min(n, rows - at))]
        assert torch.equal(out.cpu(), want)


def _attend(r, table, lengths, news, group, causal=True, window=0, scale=None, max_queries=None, max_length=None, seed=50,
            check_rest=True, cache=None):
    """Runs the kernel on the whole batch and holds every sequence against the reference."""
    q_heads, dim = r.heads * group, r.dim
    scale = dim ** -0.5 if scale is None else scale
    rows = sum(news)
    # q as a column range of a wider projection
    wide = _bf16(seed, rows + 2, (q_heads + 1) * dim)
    dev = wide.cuda()
    q, dq = (t[:, dim:].view(rows + 2, q_heads, dim) for t in (wide, dev))
    starts = torch.tensor([1] + news, dtype=torch.int32).cumsum(0, dtype=torch.int32)      # the first and last rows are nobody's
    out = torch.full((rows + 2, q_heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + 2, q_heads), 9.0, device="cuda")
    max_queries = max_queries or max(max(news), 1)
    max_length = max_length or max(max(lengths), 1)
    cache = cache or r.device()
    work = eq.alloc_cache_attention_workspace(cache, rows + 2, q_heads, len(lengths), max_queries, max_length)
    work.fill_(0xFF)                                                        # all NaN: nothing in it needs clearing
    eq.equarx_cache_attention(cache, dq, starts.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), out,
                              scale, max_queries, max_length, causal, window, lse, work)
    got, got_lse = out.double().cpu(), lse.double().cpu()
    assert (got[0] == 9).all() and (got[-1] == 9).all() and (got_lse[0] == 9).all() and (got_lse[-1] == 9).all()
    at = 1
    for b, (n, new) in enumerate(zip(lengths, news)):
        want, want_lse, mass, size = ref.attention(r, q[at:at + new].double(), table[b].tolist(), n, scale, causal, window)
        here, here_lse = got[at:at + new], got_lse[at:at + new]
        at += new
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(here), nan), b
        e = (dim + 8) * 2.0 ** -23 * size + 2.0 ** -20 + (n + 64) * 2.0 ** -23
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.02 * e[..., None]) * mass * (1 + 2.0 ** -8)
        assert ((here - want).abs()[~nan] <= bound[~nan]).all(), (b, n, new)
        empty = torch.isneginf(want_lse)
        assert torch.equal(torch.isneginf(here_lse), empty) and (here[empty] == 0).all()
        fine = ~empty & ~torch.isnan(want_lse)
        assert ((here_lse - want_lse).abs()[fine] <= (1.01 * e + 2.0 ** -21 * want_lse.abs())[fine]).all(), b
    return out, lse


@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("group", (1, 4, 5, 16, 17, 40))
def test_single_tokens(dim, block, group):
    lengths = [1, 15, 16, 63, 64, 65, 200, 0]
    r, table = _filled(11, lengths, 16, 2, dim, block)
    _attend(r, table, lengths, [1] * len(lengths), group)


@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("news", ([5, 0, 33, 7], [70, 130, 1, 64]))
def test_chunks_of_queries(dim, block, news):
    lengths = [5, 40, 33, 6] if news[0] == 5 else [100, 130, 1, 63]         # the last has more queries than tokens
    r, table = _filled(13, lengths, 64, 2, dim, block)
    for group in (1, 3):
        _attend(r, table, lengths, news, group)


@pytest.mark.parametrize("causal,window", ((False, 0), (True, 1), (True, 20), (True, 100), (True, 5000)))
@pytest.mark.parametrize("news", ([1, 1, 1], [3, 8, 2], [50, 90, 20]))
def test_masks(causal, window, news):
    lengths = [150, 90, 300]
    r, table = _filled(17, lengths, 32, 2, 128, 64)
    _attend(r, table, lengths, news, 2, causal, window)


@pytest.mark.parametrize("max_length", (1, 64, 700, 4096, 100000))
def test_any_hint_gives_the_same_within_the_bound(max_length):
    """What the host knows of the lengths sizes the launch only: short of the truth, or far above it."""
    lengths = [700, 3, 1500]
    r, table = _filled(19, lengths, 64, 1, 64, 64)
    for max_queries, news in ((1, [1, 1, 1]), (1, [20, 3, 9]), (40, [20, 3, 40])):
        _attend(r, table, lengths, news, 4, max_queries=max_queries, max_length=max_length)


def test_many_splits():
    lengths = [20000]
    r, table = _filled(23, lengths, 128, 1, 128, 128)
    _attend(r, table, lengths, [1], 8)
    _attend(r, table, lengths, [2], 8, window=300)


def test_large_scores():
    """Scores of a few hundred: one token takes nearly all."""
    lengths = [333, 90]
    r, table = _filled(29, lengths, 16, 2, 64, 64)
    _attend(r, table, lengths, [2, 1], 4, scale=4.0)
    _attend(r, table, lengths, [2, 1], 4, scale=-1.0)


@pytest.mark.parametrize("news", ([1, 2], [60, 100]))
def test_what_a_row_does_not_see_may_be_anything(news):
    """NaN in tokens behind the causal line or before the window, in slots beyond a sequence's end, in pages of others."""
    lengths = [100, 170]
    r, table = _filled(31, lengths, 48, 2, 128, 64, spare=3)
    for i in (0, 1):
        used = torch.cat([r.slots_of(table[b].tolist(), n) for b, n in enumerate(lengths)])
        rest = torch.ones(r.pages * r.page, dtype=torch.bool)
        rest[used] = False
        r.scales[i][rest] = float("nan")
        r.codes[i][rest] = 77
        r.scales[i][r.slots_of(table[1].tolist(), 170)[5]] = float("nan")   # out of every window below
    _attend(r, table, lengths, news, 3, window=64)
    r.scales[1][r.slots_of(table[0].tolist(), 100)[70]] = float("nan")      # seen by some rows: NaN there, nowhere else
    _attend(r, table, lengths, news, 3, window=64)


def test_an_infinite_or_missing_key_is_not_hidden():
    r, table = _filled(37, [30], 16, 1, 64, 64)
    r.scales[0][r.slots_of(table[0].tolist(), 30)] = float("nan")           # every score is NaN: so is the output
    _attend(r, table, [30], [1], 2)


def test_pages_that_do_not_exist_hold_no_tokens():
    lengths = [200, 40]
    r, table = _filled(41, lengths, 16, 2, 128, 128)
    table[0, 3], table[0, 7] = -1, r.pages + 5
    table[1, :] = -7                                                        # nothing at all
    _attend(r, table, lengths, [1, 1], 4)
    _attend(r, table, lengths, [20, 3], 4)


def test_lengths_beyond_the_table_end_with_it():
    r, table = _filled(43, [64], 16, 1, 64, 64)
    cache = r.device()
    q = _bf16(1, 1, 2, 64).cuda()
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    results = []
    for n in (64, 1 << 30):
        out = torch.empty_like(q)
        eq.equarx_cache_attention(cache, q, starts, table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), out, 0.1, 1, 64)
        results.append(out)
    assert torch.equal(*results)
    out = torch.full_like(q, 9.0)
    eq.equarx_cache_attention(cache, q, starts, table.cuda(), torch.tensor([-5], dtype=torch.int32, device="cuda"), out, 0.1, 1, 64)
    assert (out == 0).all()


def test_written_then_attended_on_another_stream_and_in_a_graph():
    """A decode step, captured: write the new token, attend; replayed with new tokens between eager steps."""
    r, table = _filled(47, [65, 32], 16, 2, 128, 64)
    cache = r.device()
    table, lengths = table.cuda(), torch.tensor([65, 32], dtype=torch.int32, device="cuda")
    slots = torch.tensor([int(r.slots_of(table[b].tolist(), n)[-1]) for b, n in enumerate((65, 32))], device="cuda")
    starts = torch.arange(3, dtype=torch.int32, device="cuda")
    q, k, v = _bf16(1, 2, 6, 128).cuda(), _bf16(2, 2, 2, 128).cuda(), _bf16(3, 2, 2, 128).cuda()
    out = torch.zeros(2, 6, 128, dtype=torch.bfloat16, device="cuda")
    work = eq.alloc_cache_attention_workspace(cache, 2, 6, 2, 1, 1024)

    def step():
        eq.equarx_cache_write(cache, k, v, slots)
        eq.equarx_cache_attention(cache, q, starts, table, lengths, out, 0.1, 1, 1024, workspace=work)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (60, 70, 80):
        q.copy_(_bf16(seed, 2, 6, 128)), k.copy_(_bf16(seed + 1, 2, 2, 128)), v.copy_(_bf16(seed + 2, 2, 2, 128))
        step()
        torch.cuda.synchronize()
        want = out.clone()
        assert not torch.equal(want, first)
        out.zero_()
        cache.k_codes[slots // 16, :, slots % 16] = 0
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_more_workgroups_than_are_held_at_once():
    """70 sequences of 8 heads: launched sequence after sequence."""
    lengths = [35 + 11 * (i % 9) for i in range(70)]
    r, table = _filled(31, lengths, 16, 8, 64, 64)
    _attend(r, table, lengths, [33 + i % 3 for i in range(70)], 1)
