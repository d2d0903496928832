"""Cache attention whose scores are minus infinity: a query with an infinity, or a product that overflows.

A row all of whose visible tokens have the score -inf is 0 / 0: its output is NaN and its log sum of exponentials -inf.  Where
some token's score is finite the others' weight is 0, and only a row that sees no token at all is zeros.  One element of a query
is infinite (or as large as bf16 goes, against keys as large); the codes there choose the sign of a token's score, and the others'
are 0 or finite, so that scores are -inf or what the other elements give, never NaN by the product itself."""
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu
INF = float("inf")


def _cache(lengths, page, heads, dim, block, down):
    """Keys whose element 0 is negative where down says so; there q's infinity makes the score -inf.  Elsewhere that
    element cannot be 0 (inf * 0 is NaN): such tokens are in sequences whose q is finite, or hidden."""
    counts = [-(-n // page) for n in lengths]
    r = ref.CacheRef(sum(counts), heads, page, dim, block)
    table = torch.full((len(lengths), max(counts + [1])), -1, dtype=torch.int32)
    at = 0
    for b, (n, c) in enumerate(zip(lengths, counts)):
        table[b, :c] = torch.arange(at, at + c)
        at += c
        g = torch.Generator().manual_seed(b)
        k, v = (torch.randn(n, heads, dim, generator=g) for _ in "kv")
        k[..., 0] = torch.where(down(b, torch.arange(n))[:, None], -4.0, 4.0)
        r.write(k.to(torch.bfloat16), v.to(torch.bfloat16), r.slots_of(table[b].tolist(), n))
    return r, table


def _run(r, table, lengths, news, group, q, causal, window, max_length):
    rows, heads = sum(news), r.heads * group
    starts = torch.tensor([0] + news, dtype=torch.int32).cumsum(0, dtype=torch.int32)
    out = torch.full((rows, heads, r.dim), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows, heads), 9.0, device="cuda")
    cache = r.device()
    work = eq.alloc_cache_attention_workspace(cache, rows, heads, len(lengths), max(news), max_length)
    work.fill_(0xFF)
    eq.equarx_cache_attention(cache, q.cuda(), starts.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), out,
                              r.dim ** -0.5, max(news), max_length, causal, window, lse, work)
    return out.cpu(), lse.cpu()


def _near(out, lse, wanted, n):
    """Half a bf16 unit of the result; products held to 2^-16, of sums of them; scores off by e, n tokens summed."""
    want, want_lse, mass, size = wanted
    e = (want.shape[-1] + 8) * 2.0 ** -23 * size + 2.0 ** -20 + (n + 64) * 2.0 ** -23
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2.02 * e[..., None]) * mass).all()
    assert ((lse.double() - want_lse).abs() <= 1.01 * e + 2.0 ** -21 * want_lse.abs()).all()


# What a call goes by: few rows of short sequences, few rows of any (their parts joined by four waves a row, or of many sequences by
# one), many rows, many rows in splits (joined by one wave, or by four).
FORMS = {"short": ([70, 9], 1, 64), "shares": ([5000, 700], 1, 5000), "shares of many": ([600] + [20] * 259, 1, 600),
         "rows": ([200, 90], 40, 256), "splits": ([1500], 40, 2048), "many splits": ([6000], 40, 6000)}


@pytest.mark.parametrize("dim,block", ((64, 64), (128, 64), (256, 256)))
@pytest.mark.parametrize("form", sorted(FORMS))
def test_every_score_minus_infinity(form, dim, block):
    """All a row sees is at -inf: NaN, and lse -inf.  The rows of the other heads are finite."""
    lengths, new, max_length = FORMS[form]
    group, heads = 2, 2
    r, table = _cache(lengths, 16, heads, dim, block, lambda b, t: t >= 0)
    news = [min(new, n) for n in lengths]
    q = torch.randn(sum(news), heads * group, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    q[:, 1, 0] = INF
    q[:, 1, 1:] = 0                     # codes are finite: 0 each
    q[:, 2, 0] = 3e38                   # a score beyond fp32 and no infinity in q
    out, lse = _run(r, table, lengths, news, group, q, True, 0, max_length)
    assert torch.isnan(out[:, 1]).all() and torch.isneginf(lse[:, 1]).all()
    assert torch.isnan(out[:, 2]).all() and torch.isneginf(lse[:, 2]).all()
    at = 0
    for b, (n, new) in enumerate(zip(lengths, news)):
        rows, others = slice(at, at + new), [0, 3]
        at += new
        _near(out[rows, others], lse[rows, others], ref.attention(r, q[rows, others].double(), table[b].tolist(), n, dim ** -0.5, True, 0), n)


@pytest.mark.parametrize("dim,block", ((64, 64), (128, 64), (256, 256)))
@pytest.mark.parametrize("form", sorted(FORMS))
def test_some_scores_minus_infinity(form, dim, block):
    """Tokens at -inf first, last, or in whole tiles between have weight 0: the others' answer, not NaN.  The score of a token is
    -inf by an overflow: a key of 2^100 times its size against q's largest."""
    lengths, new, max_length = FORMS[form]
    group, heads = 2, 1
    n = lengths[0]
    keep = (torch.arange(n) >= n - 3) | (torch.arange(n) == n // 2)
    r, table = _cache(lengths, 16, heads, dim, block, lambda b, t: ~keep[:len(t)] if b == 0 else t >= 0)
    slots = r.slots_of(table[0].tolist(), n)
    r.codes[0][slots, :, 0] = torch.where(keep, 0, -127).to(torch.int8)[:, None]
    r.scales[0][slots[~keep]] = 2.0 ** 100
    news = [min(new, 2 if new > 1 else 1, m) for m in lengths]
    news[0] = min(new, n)
    q = torch.randn(sum(news), heads * group, dim, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    q[:news[0], :, 0] = 3e38
    out, lse = _run(r, table, lengths, news, group, q, False, 0, max_length)
    few = ref.CacheRef(1, heads, 16, dim, block)
    for i in (0, 1):
        few.codes[i][:4], few.scales[i][:4] = r.codes[i][slots[keep]], r.scales[i][slots[keep]]
    _near(out[:news[0]], lse[:news[0]], ref.attention(few, q[:news[0]].double(), [0], 4, dim ** -0.5, False, 0), n)


@pytest.mark.parametrize("form", sorted(FORMS))
def test_minus_infinity_in_masked_tiles(form):
    """With a causal line and a window through a tile, rows whose visible tokens are all at -inf are NaN and rows that see a finite one
    are not; a row before every token sees nothing and is zeros."""
    lengths, new, max_length = FORMS[form]
    lengths, new = lengths[:1], max(new, 2)
    n, window = lengths[0], 5
    new = min(new, 20)
    keep = torch.arange(n) >= n - 1                 # only the last token is finite, for q's infinite element has a 0 there
    r, table = _cache(lengths, 16, 1, 64, 64, lambda b, t: t >= 0)
    slots = r.slots_of(table[0].tolist(), n)
    r.codes[0][slots, :, 0] = torch.where(keep, 0, -127).to(torch.int8)[:, None]
    r.scales[0][slots[~keep]] = 2.0 ** 100
    q = torch.zeros(new, 2, 64, dtype=torch.bfloat16)
    q[:, 0, 0] = 3e38
    q[:, 1, 1] = 1.0
    out, lse = _run(r, table, lengths, [new], 2, q, True, window, max_length)
    assert torch.isnan(out[:-1, 0]).all() and torch.isneginf(lse[:-1, 0]).all()
    assert torch.isfinite(out[-1, 0]).all() and torch.isfinite(lse[-1, 0])
    value = (r.codes[1][slots[-1]].double() * r.scales[1][slots[-1]].double()).view(-1)
    assert ((out[-1, 0].double() - value).abs() <= (2.0 ** -8 + 2.0 ** -15) * value.abs()).all()
    # more queries than tokens: the first ones stand before the first token
    r2, table2 = _cache([3], 16, 1, 64, 64, lambda b, t: t >= 0)
    q = torch.zeros(new, 2, 64, dtype=torch.bfloat16)
    q[:, :, 0] = INF
    rows = max(new, 4)
    q = q[:1].expand(rows, 2, 64).contiguous()
    out, lse = _run(r2, table2, [3], [rows], 2, q, True, 0, max_length)
    assert (out[:rows - 3] == 0).all() and torch.isnan(out[rows - 3:]).all() and torch.isneginf(lse).all()
