"""Performance cases of the operators around a served layer's products and attention: root-mean-square norm with the
residual's addition, of a tensor and of the partial sums that a reduction adds; low-rank adapters of many requests beside a
shared projection; and the page tables and slot maps that a key/value cache is written and read by.

A case names an operator and its sizes.  `prepare` makes what a serving program has in hand before the call -- activations,
the residual stream, weights, adapters, a pool of pages in use, output buffers and workspaces --, `run` makes the calls.
The plain forms are elementary torch operations in 32 bits (a row's mean square in 64, since the quantized forms' borders
are decided by its last bits), `exact` restates the definitions in 64 bits.

Formats.  int8: codes with one fp32 scale, largest magnitude / 127, for every `block` elements of a row.  Microscaled 4-bit
(mx4): 32 elements of a row share the scale 2^(s-127); an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.
"""
import math

import torch

own = False

MX4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


def listed():
    return [
        # One token between two layers of the 27B-shaped model: latency.
        dict(name="norm_token", op="norm", rows=1, cols=5376, gap=0, residual=True, form="bf16", block=0, dist="normal"),
        # A decode batch whose normed rows go to a 4-bit product: packed by the norm, then read back.
        dict(name="norm_decode_mx4", op="norm", rows=64, cols=5376, gap=0, residual=True, form="mx4", block=0, dist="outliers"),
        # The heads of a fused projection's queries, normed one by one: short rows, a column range of a wider tensor.
        dict(name="norm_heads", op="norm", rows=65536, cols=128, gap=64, residual=False, form="bf16", block=0, dist="normal"),
        # A prefill activation as a sequence-parallel gather sends it: normed rows in int8, then read back.
        dict(name="norm_prefill_int8", op="norm", rows=4096, cols=5376, gap=0, residual=True, form="int8", block=256, dist="outliers"),
        # A decode step's partial sums of 16 shards, reduced, added to the residual stream and normed.
        dict(name="reduced_decode", op="reduced", P=16, rows=64, cols=5376, wire=128, residual=True, form="bf16", block=0, dist="normal"),
        # The 27B-shaped prefill reduction of 8 shards, with the norm of the next layer.
        dict(name="reduced_prefill", op="reduced", P=8, rows=4096, cols=5376, wire=256, residual=True, form="bf16", block=0, dist="outliers"),
        # One token with an adapter on its joint q, k, v projection: latency.
        dict(name="adapters_token", op="adapters", M=1, K=4096, widths="4096,2048,2048", rank=16, adapters=32, order="mixed"),
        # A decode batch of 64 requests with 32 adapters among them.
        dict(name="adapters_decode", op="adapters", M=64, K=5376, widths="4096,2048,2048", rank=16, adapters=32, order="mixed"),
        # Nothing fits a tile: odd sizes, requests in no order, some without an adapter.
        dict(name="adapters_ragged", op="adapters", M=333, K=1511, widths="1001,1500", rank=24, adapters=7, order="mixed"),
        # Prompts of 4096 tokens of four requests, each with its adapter.
        dict(name="adapters_prefill", op="adapters", M=4096, K=5376, widths="5376", rank=64, adapters=4, order="grouped"),
        # A decode step of 256 sequences: five drafted tokens each are taken back to those accepted, then one more token.
        dict(name="pages_decode", op="pages", seqs=256, new=1, longest=8192, page=16, back=5),
        # 48 prompts of up to 4096 tokens enter in the place of sequences that have ended.
        dict(name="pages_prompts", op="pages", seqs=48, new=4096, longest=4096, page=64, back=4096),
    ]


WIDTHS = (512, 1024, 2048, 2560, 3840, 4096, 5376, 8192)


def _spread(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def _width(rng, lo, hi, odd=True):
    """A layer's width, or any odd one."""
    wide = [w for w in WIDTHS if lo <= w <= hi]
    return rng.choice(wide) if wide and (not odd or rng.random() < 0.5) else (_spread(rng, lo, hi) - 1) | 1


def _tokens(rng, hi):
    return min(hi, rng.choice([1 << rng.randint(0, hi.bit_length() - 1), (_spread(rng, 1, hi) - 1) | 1]))


def draw(rng):
    op = rng.choice(["norm", "norm", "reduced", "adapters", "adapters", "pages"])
    if op in ("norm", "reduced"):
        form = rng.choice(["bf16", "bf16", "int8", "mx4"])
        block = rng.choice([32, 64, 128, 256, 512]) if form == "int8" else 0
        wire = rng.choice([32, 64, 128, 256]) if op == "reduced" else 1
        P = rng.choice([2, 3, 4, 8, 16]) if op == "reduced" else 1
        most = 4096 * 5376 * 8 // P if op == "reduced" else 4096 * 5376
        rows = _tokens(rng, 16384)
        if max(block, wire) > 1:                                # whole blocks a row
            unit = max(block, wire)
            cols = unit * max(1, _spread(rng, 1, min(16384, most // rows) // unit or 1))
        else:
            cols = _width(rng, 33, min(16384, most // rows))
        residual = rng.random() < 0.75
        dist = rng.choice(["normal", "outliers"])
        if op == "norm":
            return dict(op=op, rows=rows, cols=cols, gap=rng.choice([0, 0, 8, 5, cols]), residual=residual, form=form, block=block, dist=dist)
        return dict(op=op, P=P, rows=rows, cols=cols, wire=wire, residual=residual, form=form, block=block, dist=dist)
    if op == "adapters":
        M = _tokens(rng, 4096)
        count = rng.choice([1, 2, 3])
        widths = [_width(rng, 65, 5376 // count) for _ in range(count)]
        rank = rng.choice([8, 16, 24, 32, 64])
        adapters = _spread(rng, 1, 32)
        adapters = max(1, min(adapters, 4096 * 4 * 64 // (M * rank * count)))
        return dict(op=op, M=M, K=_width(rng, 65, 5376), widths=",".join(map(str, widths)), rank=rank, adapters=adapters,
                    order=rng.choice(["grouped", "mixed"]))
    page = rng.choice([16, 32, 64, 128])
    if rng.random() < 0.5:                                      # single tokens, or a few drafted ones
        new, back = rng.choice([1, 1, 2, 5]), rng.choice([0, 1, 5])
        longest = _spread(rng, 16, 16384)
        seqs = min(_spread(rng, 1, 1024), 256 * 8192 // longest)
    else:
        longest = _spread(rng, 16, 8192)
        new, back = longest, longest
        seqs = min(_spread(rng, 1, 256), 48 * 4096 // longest)
    return dict(op=op, seqs=max(1, seqs), new=new, longest=longest, page=page, back=back)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 41)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols, gap, dist, factor=None):
    """bf16 [rows, cols], a column range of a tensor that is `gap` columns wider; per-token factors and a few channels
    fifty times larger where dist is "outliers"."""
    v = _randn(g, rows, cols)
    if dist == "outliers":
        v *= torch.exp(_randn(g, rows, 1)) if factor is None else factor
        channels = torch.randperm(cols, generator=g, device="cuda")[:max(1, round(0.001 * cols))]
        v[:, channels] *= 50.0
    wide = torch.zeros((rows, cols + gap), dtype=torch.bfloat16, device="cuda")
    wide[:, :cols] = v.to(torch.bfloat16)
    return wide[:, :cols]


def _widths(case):
    return [int(w) for w in case["widths"].split(",")]


def _ids(case, seed):
    """int32 [M] on the host: the adapter of every row, -1 for none (one row in sixteen, where there are many)."""
    g = torch.Generator().manual_seed(seed * 13 + 7)
    M, adapters = case["M"], case["adapters"]
    ids = torch.randint(0, adapters, (M,), generator=g)
    if M >= 16:
        ids[torch.rand(M, generator=g) < 1 / 16] = -1
    if case["order"] == "grouped":                              # prompts one after the other
        ids = ids.sort().values
    return ids.to(torch.int32)


def _plan(case):
    """Lengths before the pass, tokens kept of them, and new ones; int64 on the host, the same for every seed."""
    g = torch.Generator().manual_seed(5)
    n, longest, new = case["seqs"], case["longest"], case["new"]
    u = torch.rand(n, generator=g)
    if new < longest:                                           # sequences that go on
        kept = (u * (longest - new + 1)).long()
        had = torch.minimum(kept + torch.randint(0, case["back"] + 1, (n,), generator=g), torch.tensor(longest))
        counts = torch.full((n,), new)
    else:                                                       # sequences that make room for others
        had = (torch.rand(n, generator=g) * (longest + 1)).long()
        kept = torch.zeros(n, dtype=torch.long)
        counts = 1 + (u * longest).long().clamp(max=longest - 1)
        counts[0] = longest
    return had, kept, counts


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    st = dict(op=op, case=case)
    if op in ("norm", "reduced"):
        rows, cols = case["rows"], case["cols"]
        if op == "norm":
            st["x"] = _activations(g, rows, cols, case["gap"], case["dist"])
        else:
            factor = torch.exp(_randn(g, rows, 1))              # a row is large in all of its partial sums
            st["partials"] = [_activations(g, rows, cols, 0, case["dist"], factor) for _ in range(case["P"])]
        st["weight"] = (1.0 + 0.1 * _randn(g, cols)).to(torch.bfloat16)
        st["residual"] = (4.0 * _randn(g, rows, cols)).to(torch.bfloat16) if case["residual"] else None
    elif op == "adapters":
        M, K, rank, widths = case["M"], case["K"], case["rank"], _widths(case)
        st["x"] = _randn(g, M, K).to(torch.bfloat16)
        st["a"] = (_randn(g, case["adapters"], len(widths) * rank, K) * K ** -0.5).to(torch.bfloat16)
        st["b"] = (_randn(g, case["adapters"], sum(widths), rank) * rank ** -0.5).to(torch.bfloat16)
        st["factors"] = 0.5 + torch.rand(case["adapters"], generator=g, device="cuda")
        st["ids"] = _ids(case, seed).cuda()
        st["out"] = _randn(g, M, sum(widths)).to(torch.bfloat16)        # the shared projection's outputs
    else:
        had, kept, counts = _plan(case)
        page, n = case["page"], case["seqs"]
        width = -(-case["longest"] // page)
        held = -(-had // page)
        total = int(torch.maximum(held, -(-(kept + counts) // page)).sum()) + 3
        order = torch.randperm(total, generator=torch.Generator().manual_seed(seed * 17 + 3)).int()
        at = held.cumsum(0) - held
        i = torch.arange(width)
        st["table"] = torch.where(i < held[:, None], order[(at[:, None] + i).clamp(max=total - 1)], -1).int().cuda()
        used = int(held.sum())
        free = torch.full((total,), -1, dtype=torch.int32)
        free[:total - used] = order[used:]
        st["free"], st["free_count"] = free.cuda(), torch.tensor([total - used], dtype=torch.int32).cuda()
        on = lambda t: t.to(torch.int32).cuda()
        st["lengths"], st["keep"], st["counts"] = on(had), on(kept), on(counts)
        st["tags"] = torch.arange(n, dtype=torch.int32, device="cuda") % 7 - 1
        st["rows"] = int(counts.sum()) + 5                      # as a captured step has them: not all are used
    if own:
        _prepare_own(st, case)
    return st


def _prepare_own(st, case):
    """The plan of a program that uses the library: output buffers and workspaces."""
    from paper_2506_17615_amd import binding as eq
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")
    if case["op"] in ("norm", "reduced"):
        rows, cols = case["rows"], case["cols"]
        st["out"] = empty(rows, cols)
        if case["form"] == "int8":
            st["codes"] = empty(rows, cols, dtype=torch.int8)
            st["scales"] = empty(rows, cols // case["block"], dtype=torch.float32)
        elif case["form"] == "mx4":
            st["packed"] = eq.alloc_mx4(rows, cols)
    elif case["op"] == "adapters":
        widths = _widths(case)
        st["slice_ends"] = tuple(sum(widths[:i + 1]) for i in range(len(widths)))
        st["workspace"] = eq.alloc_adapters_workspace(case["M"], sum(widths), case["K"], case["rank"], len(widths), case["adapters"])
    else:
        st["pages"] = eq.Pages(st["table"], st["lengths"], st["free"], st["free_count"])
        ints = lambda n, dtype=torch.int32: torch.empty(n, dtype=dtype, device="cuda")
        st["q_starts"], st["granted"] = ints(case["seqs"] + 1), ints(case["seqs"])
        st["slots"], st["positions"], st["row_tags"] = ints(st["rows"], torch.int64), ints(st["rows"]), ints(st["rows"])


# ---------------------------------------------------------------- one pass

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2506_17615_amd import binding as eq
    op, case = st["op"], st["case"]
    if op in ("norm", "reduced"):
        form = case["form"]
        outputs = {}
        if form == "bf16":
            outputs = dict(out=st["out"])
        elif form == "int8":
            outputs = dict(codes=st["codes"], scales=st["scales"], codes_block=case["block"])
        else:
            outputs = dict(mx4_codes=st["packed"][0], mx4_scales=st["packed"][1])
        if op == "norm":
            eq.equarx_norm(st["x"], st["weight"], EPS, st["residual"], **outputs)
        else:
            eq.equarx_norm_reduced(st["partials"], case["wire"], st["weight"], EPS, st["residual"], **outputs)
        if form == "int8":
            eq.equarx_dequantize(st["codes"], st["scales"], case["block"], st["out"])
        elif form == "mx4":
            eq.equarx_mx4_dequantize(*st["packed"], st["out"])
        return st["out"] if st["residual"] is None else (st["out"], st["residual"])
    if op == "adapters":
        eq.equarx_adapters(st["x"], st["a"], st["b"], st["factors"], st["ids"], st["out"], st["slice_ends"], st["workspace"])
        return st["out"]
    eq.equarx_pages_trim(st["pages"], case["page"], st["keep"])
    eq.equarx_pages_extend(st["pages"], case["page"], st["counts"], st["q_starts"], st["slots"], st["granted"], st["positions"],
                           st["tags"], st["row_tags"])
    return (st["q_starts"], st["slots"], st["granted"], st["positions"], st["row_tags"], st["table"], st["lengths"], st["free_count"])


def _chain(partials, block):
    """The quantized chain over partial sums: every running sum to int8 and back, in array order."""
    shape = partials[0].shape
    v = partials[0].float().view(-1, block)
    for p in list(partials[1:]) + [None]:
        codes, scale = _codes(v)
        v = codes * scale
        if p is not None:                                       # one rounding for product and sum: both are exact in 64 bits
            v = (codes.double() * scale.double() + p.double().view(-1, block)).float()
    return v.view(shape).to(torch.bfloat16)


def _codes(v):
    """[..., block] fp32 -> codes (as fp32) and scales [..., 1]."""
    top = v.abs().amax(dim=-1, keepdim=True)
    alive = top >= 127.0 * 2.0 ** -126
    most = torch.full_like(top, 127.0)                          # by tensors: a number is multiplied by as its reciprocal
    scale = torch.where(alive, top / most, 0.0)
    inverse = torch.where(alive, most / torch.where(alive, top, 1.0), 0.0)
    return torch.round(v * inverse), scale


def _nearest_values(x):
    """A tensor of rows as the values that its packed 4-bit form stands for, fp32."""
    rows, cols = x.shape
    padded = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float32, device=x.device)
    padded[:, :cols] = x
    v = padded.view(rows, -1, 32)
    top = v.abs().amax(dim=-1, keepdim=True)
    _, e = torch.frexp(top)
    s = torch.where(top > 0, e - 3, -127).clamp(min=-127)
    a = torch.ldexp(v, -s)
    m = a.abs()
    fine = torch.where(m < 2, torch.round(m * 2) / 2, torch.where(m < 4, torch.round(m), torch.round(m / 2) * 2))
    return torch.ldexp(torch.copysign(fine.clamp(max=6.0), a), s).view(rows, -1)[:, :cols]


def _run_plain(st):
    op, case = st["op"], st["case"]
    if op in ("norm", "reduced"):
        h = st["x"] if op == "norm" else _chain(st["partials"], case["wire"])
        if st["residual"] is not None:
            h = st["residual"].copy_(h.float() + st["residual"].float())
        mean = h.double().square().mean(dim=-1, keepdim=True)
        y = h.float() * (1.0 / torch.sqrt(mean + EPS)).float() * st["weight"].float()
        if case["form"] == "int8":
            codes, scale = _codes(y.view(-1, case["block"]))
            y = (codes * scale).view(h.shape)
        elif case["form"] == "mx4":
            y = _nearest_values(y)
        out = y.to(torch.bfloat16)
        return out if st["residual"] is None else (out, st["residual"])
    if op == "adapters":
        return _adapters_plain(st, case)
    return _pages_plain(st, case)


def _adapters_plain(st, case):
    """All adapters' products, of which every row keeps its own's."""
    M, rank, adapters = case["M"], case["rank"], case["adapters"]
    ids = st["ids"].long()
    mine = ids.unsqueeze(1) == torch.arange(adapters, device="cuda")                    # none for -1
    t = torch.matmul(st["x"].float(), st["a"].float().view(-1, case["K"]).t()).view(M, adapters, -1)
    t = t * (mine * st["factors"]).unsqueeze(-1)
    at, parts = 0, []
    for s, width in enumerate(_widths(case)):
        b = st["b"][:, at:at + width].float().transpose(1, 2).reshape(adapters * rank, width)
        parts.append(torch.matmul(t[:, :, s * rank:(s + 1) * rank].reshape(M, -1), b))
        at += width
    st["out"].copy_(st["out"].float() + torch.cat(parts, dim=1))
    return st["out"]


def _pages_plain(st, case):
    page, table, lengths, free = case["page"], st["table"], st["lengths"], st["free"]
    width = table.shape[1]
    up = lambda n: torch.div(n + (page - 1), page, rounding_mode="floor")
    at = torch.arange(width, device="cuda")
    # back to the tokens kept: pages behind them go to the stack, sequence by sequence
    kept = torch.minimum(lengths, st["keep"])
    gone = (at >= up(kept)[:, None]) & (at < up(lengths)[:, None])
    place = st["free_count"] + gone.flatten().cumsum(0) - 1
    free = torch.cat((free, free[:1])).scatter_(0, torch.where(gone.flatten(), place, free.numel()), table.flatten())[:-1]
    count = st["free_count"] + gone.sum()
    table = torch.where(gone, -1, table)
    # new tokens: pages from the top of the stack, in order of the sequences
    counts = st["counts"].long()
    fits = kept + counts <= width * page
    wanted = torch.where(fits, counts, 0)
    wanted = torch.where(wanted.cumsum(0) <= st["rows"], wanted, 0)
    need = up(kept + wanted) - up(kept)
    upto = need.cumsum(0)
    granted = torch.where((upto <= count) | (need == 0), wanted, 0)
    need = up(kept + granted) - up(kept)
    first = need.cumsum(0) - need
    j = at - up(kept)[:, None]
    taken = (j >= 0) & (j < need[:, None])
    top = (count - 1 - first[:, None] - j).clamp(min=0, max=free.numel() - 1)
    table = torch.where(taken, free[top], table).int()
    # rows of the step
    starts = torch.cat((torch.zeros_like(granted[:1]), granted.cumsum(0)))
    row = torch.arange(st["rows"], device="cuda")
    b = (torch.searchsorted(starts, row, right=True) - 1).clamp(max=case["seqs"] - 1)
    real = row < starts[-1]
    t = kept[b] + row - starts[b]
    entry = table[b, torch.div(t, page, rounding_mode="floor").clamp(max=width - 1)].long()
    slots = torch.where(real, entry * page + t % page, -1)
    st["table"].copy_(table)
    st["lengths"].copy_(kept + granted)
    st["free"].copy_(free)
    st["free_count"].copy_(count - need.sum())
    return (starts.int(), slots, granted.int(), torch.where(real, t, -1).int(), torch.where(real, st["tags"][b], -1).int(), st["table"],
            st["lengths"], st["free_count"])


# ---------------------------------------------------------------- the definitions in 64 bits

def _int8_values(v, block):
    """Nearest multiples of a block's largest magnitude / 127, 64 bits."""
    w = v.reshape(-1, block)
    unit = (w.abs().max(dim=-1, keepdim=True).values / 127).clamp(min=1e-300)
    return (torch.round(w / unit) * unit).reshape(v.shape)


def _mx4_values(x):
    """Rows in 64 bits -> the nearest of the values that 4 bits and the block's scale can hold, ties to the even code."""
    rows, cols = x.shape
    full = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    top = full.abs().max(dim=-1, keepdim=True).values
    unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2).clamp(min=2.0 ** -127)
    m = full.abs() / unit
    best, value = torch.full_like(m, math.inf), torch.zeros_like(m)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                           # even codes first: they keep a tie
        far = (m - MX4_VALUES[i]).abs()
        value = torch.where(far < best, MX4_VALUES[i], value)
        best = torch.minimum(best, far)
    return (value * torch.sign(full) * unit).reshape(rows, -1)[:, :cols]


def _reduced_values(partials, block):
    """The chain with the roundings that its definition has: sums, scales, reciprocals and products to 32 bits, codes to
    whole numbers, the result to bf16; everything else in 64."""
    total, to32 = partials[0].double(), lambda t: t.float().double()
    for i in range(len(partials)):
        w = total.reshape(-1, block)
        top = w.abs().max(dim=-1, keepdim=True).values
        alive = top >= 127 * 2.0 ** -126
        scale, inverse = to32(top / 127) * alive, to32(127 / torch.where(alive, top, 1.0)) * alive
        total = (torch.round(to32(w * inverse)) * scale).reshape(partials[0].shape)
        if i + 1 < len(partials):
            total = to32(total + partials[i + 1].double())
    return to32(total).to(torch.bfloat16).double()


def exact(case, seed):
    with_own = own
    globals()["own"] = False
    try:
        st = prepare(case, seed)
    finally:
        globals()["own"] = with_own
    op = case["op"]
    if op in ("norm", "reduced"):
        x = st["x"].double() if op == "norm" else _reduced_values(st["partials"], case["wire"])
        stream = x if st["residual"] is None else x + st["residual"].double()
        h = stream.to(torch.bfloat16).double()                   # the residual stream is kept in bf16, and its norm taken
        y = h / torch.sqrt(h.pow(2).sum(dim=1, keepdim=True) / case["cols"] + EPS) * st["weight"].double()
        if case["form"] == "int8":
            y = _int8_values(y, case["block"])
        elif case["form"] == "mx4":
            y = _mx4_values(y)
        return y if st["residual"] is None else (y, stream)
    if op == "adapters":
        out, ids, rank = st["out"].double(), st["ids"].long(), case["rank"]
        for i in range(case["adapters"]):
            rows = (ids == i).nonzero().flatten()
            if rows.numel() == 0:
                continue
            t = st["x"][rows].double() @ st["a"][i].double().T
            begin = 0
            for s, width in enumerate(_widths(case)):
                b = st["b"][i, begin:begin + width].double()
                out[rows, begin:begin + width] += float(st["factors"][i]) * (t[:, s * rank:(s + 1) * rank] @ b.T)
                begin += width
        return out
    return None                                                  # whole numbers


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Inputs read once, outputs written once.  Quantizing and reading back count as the two operators they are.
    Operations: a multiply-add is two; an add, a square-add, two multiplies for an element that is normed, five for one
    that is quantized and read, six for one that a reduction adds."""
    op = case["op"]
    if op in ("norm", "reduced"):
        rows, cols = case["rows"], case["cols"]
        n, P = rows * cols, case.get("P", 1)
        form = {"bf16": 2, "int8": 2 * (1 + 4 / max(case["block"], 1)) + 2, "mx4": 2 * 17 / 32 + 2}[case["form"]]
        flops = 5 + (0 if case["form"] == "bf16" else 5) + (6 * P if op == "reduced" else 0)
        return {"bytes": n * (2 * P + (4 if case["residual"] else 0) + form) + 2 * cols, "flops": n * flops}
    if op == "adapters":
        M, K, rank, widths = case["M"], case["K"], case["rank"], _widths(case)
        R, N = rank * len(widths), sum(widths)
        used = min(case["adapters"], M)
        return {"bytes": 2 * M * K + 2 * used * (R * K + N * rank) + 4 * M * N + 4 * M, "flops": 2 * M * (R * K + rank * N)}
    had, kept, counts = _plan(case)
    page, n = case["page"], case["seqs"]
    moved = int((-(-had // page) + -(-kept // page)).sum()) + int((-(-(kept + counts) // page) - -(-kept // page)).sum())
    rows = int(counts.sum()) + 5
    return {"bytes": 8 * moved + 16 * rows + 40 * n, "flops": 4 * rows}
