"""How near cache attention is: products of probability and value scale are held to 2^-16 of each, in every geometry and form of a call.

The inputs leave nothing else to be far off.  A query is 1 in one element and 0 elsewhere, key scales are powers of two and so is the
call's: a score is a code times a power of two, and what the kernels add to it is one rounding of log2(e) times that, below 6 in
size, 2^-23 of it; one of the difference from a reference up to 20 away, 2^-24 of that; and an exponential, 2^-22: together less
than 2^-18 of a probability.  Tokens that count are few (`count`, of which a row sees those within e^60 of its largest), each a
rounding of 2^-23 in the sums above and below the line; the others, below e^-100 of a row's largest, may be zeros: 4000 of them
with values up to 200 are 2^-100 at most.  With u = 2^-8 for the result's own rounding the bound is

    |out - want| <= u |want| + (2^-16 + 2 (2^-18 + (count + 64) 2^-23)) (1 + u) sum p |v| + 2^-100.

That a result of one bf16 a product is outside it, in every case, is held on the host, by mistakes planted in the reference."""
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq

GEOMETRIES = ((64, 64), (128, 64), (128, 128), (256, 64), (256, 128), (256, 256))
SCALE = 0.125
# form: lengths, queries of a sequence, heads, group, max_length, window.  Few rows: of short sequences; in shares, joined by four
# waves a row or (256 items and more) by one; two sixteens of rows where heads have up to 128.  Many rows: whole; in splits,
# joined by one wave or by four.
FORMS = {
    "short": ([1, 2, 5, 17, 64, 90], 1, 2, 4, 64, 0),
    "short, many heads": ([3, 40, 70], 1, 1, 24, 64, 0),
    "shares": ([3000, 65, 700], 1, 1, 4, 4096, 0),
    "shares, windows": ([3000, 650], 3, 2, 2, 4096, 300),
    "shares, many heads": ([1500, 4], 2, 1, 11, 4096, 0),
    "shares of many": ([900, 2, 70, 129] * 33, 1, 2, 3, 900, 0),
    "rows": ([90, 200, 64], 40, 2, 2, 256, 0),
    "rows, windows": ([250, 130], 50, 1, 3, 256, 33),
    "splits": ([1500, 60], 20, 1, 4, 1536, 0),
    "many splits": ([4000], 20, 1, 4, 4096, 0),
    "many splits, windows": ([4000], 24, 2, 4, 4096, 1500),
}


class Case:
    def __init__(self, form, dim, block, page=16):
        self.lengths, self.new, self.heads, self.group, self.max_length, self.window = FORMS[form]
        self.dim, self.block = dim, block
        g = torch.Generator().manual_seed(dim + block)
        counts = [-(-n // page) for n in self.lengths]
        pages = sum(counts)
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((len(counts), max(counts)), -1, dtype=torch.int32)
        r = self.cache = ref.CacheRef(pages, self.heads, page, dim, block)
        for i in (0, 1):
            r.codes[i] = torch.randint(-127, 128, r.codes[i].shape, generator=g, dtype=torch.int8)
        r.scales[0][:] = 0.25
        r.scales[1] = 0.5 + torch.rand(r.scales[1].shape, generator=g)
        self.news, at = [], 0
        for b, (n, c) in enumerate(zip(self.lengths, counts)):
            self.table[b, :c] = order[at:at + c]
            at += c
            self.news.append(min(self.new, n))
            # a few tokens count, the last ones among them; the others are 100 and more below
            far = torch.rand(n, generator=g) * n > 12
            far[-2:] = False
            slots = r.slots_of(self.table[b].tolist(), n)[far]
            r.codes[0][slots], r.scales[0][slots] = -127, 8.0
        rows = sum(self.news)
        where = torch.randint(0, dim, (rows, self.heads * self.group, 1), generator=g)
        self.q = torch.zeros(rows, self.heads * self.group, dim).scatter_(2, where, 1.0).to(torch.bfloat16)

    def answer(self, product=None):
        """out, lse, sum of p |v| and the tokens that count; `product`: what becomes of exp(s - a reference) times a value's scale."""
        outs = []
        at = 0
        for b, (n, new) in enumerate(zip(self.lengths, self.news)):
            slots = self.cache.slots_of(self.table[b].tolist(), n)
            place = torch.arange(n - new, n)[:, None]
            t = torch.arange(n)[None]
            seen = (t <= place) & (t > place - self.window) if self.window else t <= place
            q = self.q[at:at + new].double().view(new, self.heads, self.group, self.dim)
            at += new
            out, mass = torch.empty_like(q), torch.empty_like(q)
            lse, count = (torch.empty(new, self.heads, self.group, dtype=torch.float64) for _ in range(2))
            for h in range(self.heads):
                (keys, key_scales), (codes, scales) = (
                    (self.cache.codes[i][slots, h].double(), self.cache.scales[i][slots, h].double().repeat_interleave(self.block, -1)) for i in (0, 1))
                s = torch.where(seen[:, None], SCALE * (q[:, h] @ (keys * key_scales).T), -torch.inf)       # [new, group, n]
                top = s.amax(-1, keepdim=True)
                e = torch.exp(s - top)
                total = e.sum(-1, keepdim=True)
                if product is None:
                    out[:, h] = e @ (scales * codes) / total
                else:
                    near = (e > 1e-30).any(0).any(0)                                             # the others are zeros
                    out[:, h] = (product(e[..., near, None] * scales[near]) * codes[near]).sum(-2) / total
                mass[:, h] = e @ (scales * codes).abs() / total
                lse[:, h] = (top + torch.log(total)).squeeze(-1)
                count[:, h] = (s > top - 60).sum(-1)
            outs.append([x.flatten(1, 2) for x in (out, lse, mass, count)])
        return [torch.cat(x) for x in zip(*outs)]


def _rest(count):
    return 2.0 ** -18 + (count + 64) * 2.0 ** -23


def _outside(out, answer):
    want, _, mass, count = answer
    u = 2.0 ** -8
    bound = u * want.abs() + (2.0 ** -16 + 2 * _rest(count)[..., None]) * (1 + u) * mass + 2.0 ** -100
    return int(((out - want).abs() > bound).sum())


def _bf16(x):
    return x.to(torch.float32).to(torch.bfloat16).double()


def _cut(x):
    """The upper half of the fp32 pattern: what the first of two bf16 holds."""
    return (x.to(torch.float32).view(torch.int32) & -65536).view(torch.float32).double()


PLANTED = {"rounded to one": _bf16, "the first alone": _cut, "the second twice": lambda x: _cut(x) + 2 * _bf16(x - _cut(x)),
           "the second's sign": lambda x: _cut(x) - _bf16(x - _cut(x))}


@pytest.mark.parametrize("dim,block", ((64, 64), (256, 128)))
@pytest.mark.parametrize("form", sorted(FORMS))
def test_the_bound_tells_two_bf16_from_less(form, dim, block):
    case = Case(form, dim, block)
    answer = case.answer()
    assert _outside(case.answer(lambda x: _cut(x) + _bf16(x - _cut(x)))[0].to(torch.bfloat16).double(), answer) == 0
    for name, mistake in PLANTED.items():
        assert _outside(case.answer(mistake)[0].to(torch.bfloat16).double(), answer) > 0, name


@pytest.mark.gpu
@pytest.mark.parametrize("dim,block", GEOMETRIES)
@pytest.mark.parametrize("form", sorted(FORMS))
def test_products_are_held_to_what_is_promised(form, dim, block):
    case = Case(form, dim, block)
    rows, q_heads = case.q.shape[:2]
    cache = case.cache.device()
    out, lse = torch.empty(case.q.shape, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, q_heads, device="cuda")
    starts = torch.tensor([0] + case.news, dtype=torch.int32).cumsum(0, dtype=torch.int32)
    work = eq.alloc_cache_attention_workspace(cache, rows, q_heads, len(case.lengths), case.new, case.max_length)
    eq.equarx_cache_attention(cache, case.q.cuda(), starts.cuda(), case.table.cuda(), torch.tensor(case.lengths, dtype=torch.int32).cuda(),
                              out, SCALE, case.new, case.max_length, True, case.window, lse, work)
    answer = case.answer()
    assert _outside(out.double().cpu(), answer) == 0
    _, want, _, count = answer
    assert ((lse.double().cpu() - want).abs() <= 1.01 * _rest(count) + 2.0 ** -21 * (1 + want.abs())).all()
