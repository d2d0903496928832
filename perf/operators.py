"""Performance cases of the serving operators that sit beside the reduction: microscaled 4-bit numbers and their product
(the row-parallel layers whose partial sums the library reduces), and the int8 key/value cache with the attention that
reads it.

A case names an operator and its sizes.  `prepare` makes what a serving program has in hand before the call -- the
activations, the packed weights, a cache filled by earlier steps, page tables, output buffers and workspaces --, `run`
makes the calls.  The plain forms are elementary torch operations in 32 bits, `exact` restates the definitions in 64 bits.

Formats.  Microscaled 4-bit (mx4): 32 consecutive elements of a row share the scale 2^(s-127), one byte s (255: not a
number); an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, the first of a pair in a byte's low half.  Rows are
padded with zero elements to whole groups of 128 columns.  Cache: int8 codes with one fp32 scale per `block` elements
along a head's dimension, in pages of `page` tokens; keys [pages, heads, page, dim], values [pages, heads, page / 16, dim,
16], scales of both [pages, heads, dim / block, page].
"""
import math

import torch

own = False

MX4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # A decode step's activations (64 tokens x 5376) before a 4-bit product: latency.
        dict(name="mx4_rows_decode", op="mx4", rows=64, cols=5376, gap=0, dist="normal"),
        # The 27B-shaped prefill activation (4096 x 5376), one of two column shards of a wider tensor.
        dict(name="mx4_rows_prefill", op="mx4", rows=4096, cols=5376, gap=5376, dist="outliers"),
        # One token through a projection of the 27B-shaped hidden size: the weights are read and little else happens.
        dict(name="linear_token", op="linear", M=1, N=5376, K=4096, dist="normal"),
        # A decode batch of 64 tokens.
        dict(name="linear_decode", op="linear", M=64, N=5376, K=5376, dist="normal"),
        # Nothing fits a tile: an odd batch, an odd output width, a last group of columns that is not full.
        dict(name="product_ragged", op="product", M=333, N=2501, K=1511, dist="outliers"),
        # Prefill of 4096 tokens: activations quantized in the call.
        dict(name="linear_prefill", op="linear", M=4096, N=5376, K=4096, dist="outliers"),
        # The largest product, both operands packed already.
        dict(name="product_large", op="product", M=8192, N=8192, K=8192, dist="normal"),
        # A decode step of 64 short sequences: one new token each, then the sequences are read back.
        dict(name="cache_decode", op="cache", seqs=64, new=1, longest=64, heads=8, dim=128, block=128, page=16),
        # Four prompts of 4096 tokens enter the cache and are read back.
        dict(name="cache_prompt", op="cache", seqs=4, new=4096, longest=4096, heads=8, dim=128, block=64, page=64),
        # Decode of 64 sequences of very different lengths, four query heads to a key head.
        dict(name="attend_decode", op="attend", seqs=64, new=1, longest=8192, heads=8, group=4, dim=128, block=128,
             page=16, window=0),
        # One token at the end of a long context, eight query heads to a key head.
        dict(name="attend_long", op="attend", seqs=1, new=1, longest=131072, heads=4, group=8, dim=128, block=128, page=64,
             window=0),
        # A chunk of 2048 prompt tokens at the end of contexts of 8192.
        dict(name="attend_prompt", op="attend", seqs=2, new=2048, longest=8192, heads=8, group=4, dim=128, block=64,
             page=64, window=0),
    ]


WIDTHS = (512, 1024, 2048, 2560, 3840, 4096, 5376, 8192)


def _spread(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def _width(rng, lo, hi):
    """A layer's width, or any odd one."""
    wide = [w for w in WIDTHS if w <= hi]
    return rng.choice(wide) if wide and rng.random() < 0.5 else (_spread(rng, lo, hi) - 1) | 1


def _tokens(rng, hi):
    return rng.choice([1 << rng.randint(0, hi.bit_length() - 1), (_spread(rng, 1, hi) - 1) | 1])


def draw(rng):
    op = rng.choice(["mx4", "linear", "linear", "product", "cache", "attend", "attend", "attend"])
    if op == "mx4":
        rows = _tokens(rng, 4096)
        cols = _width(rng, 33, min(16384, 4096 * 5376 // rows))
        gap = rng.choice([0, 0, 8, cols])
        return dict(op=op, rows=rows, cols=cols, gap=gap, dist=rng.choice(["normal", "outliers"]))
    if op in ("linear", "product"):
        return dict(op=op, M=_tokens(rng, 8192), N=_width(rng, 65, 8192), K=_width(rng, 65, 8192), dist=rng.choice(["normal", "outliers"]))
    dim = rng.choice([64, 128, 128, 256])
    block = rng.choice([b for b in (64, 128, 256) if b <= dim])
    page = rng.choice([16, 32, 64, 128])
    heads = rng.choice([1, 2, 4, 8])
    if op == "cache":
        longest = _spread(rng, 1, 4096)
        new = rng.choice([1, longest, rng.randint(1, longest)])
        seqs = min(_spread(rng, 1, 64), max(1, 4 * 4096 * 8 * 128 // (longest * heads * dim)))
        return dict(op=op, seqs=seqs, new=new, longest=longest, heads=heads, dim=dim, block=block, page=page)
    group = rng.choice([1, 2, 4, 5, 8])
    if rng.random() < 0.6:                              # single tokens, or a few drafted ones
        new = rng.choice([1, 1, 1, 2, 5])
        most = 64 * 3584 * 8 * 128 // (heads * dim)          # tokens of all sequences together
        longest = _spread(rng, new, min(131072, most))
        seqs = min(_spread(rng, 1, 128), most // longest)
    else:                                               # a chunk of a prompt
        longest = _spread(rng, 16, 8192)
        new = rng.randint(max(1, longest // 8), min(longest, 2048))
        seqs = min(_spread(rng, 1, 8), max(1, 2 * 2048 * 8192 * 32 * 128 // (new * longest * heads * group * dim)))
    window = rng.choice([0, 0, 0, 128, 1024])
    return dict(op=op, seqs=seqs, new=new, longest=longest, heads=heads, group=group, dim=dim, block=block, page=page,
                window=window)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols, gap, dist):
    """bf16 [rows, cols], a column range of a tensor that is `gap` columns wider; per-token factors and a few channels
    fifty times larger where dist is "outliers"."""
    v = _randn(g, rows, cols)
    if dist == "outliers":
        v *= torch.exp(_randn(g, rows, 1))
        channels = torch.randperm(cols, generator=g, device="cuda")[:max(1, round(0.001 * cols))]
        v[:, channels] *= 50.0
    wide = torch.zeros((rows, cols + gap), dtype=torch.bfloat16, device="cuda")
    wide[:, :cols] = v.to(torch.bfloat16)
    return wide[:, :cols]


def _pack(x):
    """Packed codes and scale bytes of a tensor of rows, as earlier steps left them (weights: packed once, at loading)."""
    rows, cols = x.shape
    padded = torch.zeros((rows, -(-cols // 128) * 128), dtype=torch.float32, device=x.device)
    padded[:, :cols] = x
    v = padded.view(rows, -1, 32)
    s = _shared_exponent(v)
    a = torch.ldexp(v, -s)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float32, device=x.device)
    magnitude = torch.bucketize(a.abs(), edges)                  # an edge itself goes to the lower code
    for odd in (0.75, 1.75, 3.5):                                # ... and to the upper one where that is the even one
        magnitude += (a.abs() == odd)
    code = (magnitude + 8 * (a < 0)).to(torch.uint8).view(rows, -1, 2)
    return (code[..., 0] | code[..., 1] << 4).contiguous(), (s.view(rows, -1) + 127).to(torch.uint8)


def _unpack(codes, scales, cols):
    """The values that packed rows stand for, fp32 [rows, cols]."""
    rows = codes.shape[0]
    table = torch.tensor(MX4_VALUES + tuple(-v for v in MX4_VALUES), dtype=torch.float32, device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), dim=-1).long()].view(rows, -1, 32)
    return torch.ldexp(v, (scales.int() - 127).unsqueeze(-1)).view(rows, -1)[:, :cols]


def _shared_exponent(v):
    """[..., 32] -> [..., 1]: the largest magnitude's exponent less two, that of 4 and 6; -127 at least."""
    _, e = torch.frexp(v.abs().amax(dim=-1, keepdim=True))
    return torch.where(v.abs().amax(dim=-1, keepdim=True) > 0, e - 3, -127).clamp(min=-127)


def _lengths(case):
    """Tokens of every sequence, the new ones among them: from `new` to `longest`, the first sequence the longest."""
    u = torch.rand(case["seqs"], generator=torch.Generator().manual_seed(3))
    lengths = [case["new"] + int(float(r) * (case["longest"] - case["new"] + 1)) for r in u]
    lengths[0] = case["longest"]
    if case["op"] == "attend" and case["new"] > 1:
        lengths = [max(n, (case["longest"] + case["new"]) // 2) for n in lengths]
    return [min(n, case["longest"]) for n in lengths]


def _page_table(lengths, page, seed):
    """int32 [seqs, pages of the longest]: the pages of a pool, handed out in no order; and the pool's size."""
    width = -(-max(lengths) // page)
    counts = [-(-n // page) for n in lengths]
    total = sum(counts) + 1                                      # a page that nobody holds
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed * 11 + 5))
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c].int()
        at += c
    return table, total


def _slots(table, page, b, first, count):
    """Cache slots of sequence b's tokens first .. first + count - 1."""
    t = torch.arange(first, first + count)
    return table[b, t // page].long() * page + t % page


def _int8_blocks(x, block):
    """bf16 [..., dim] -> int8 codes [..., dim] and fp32 scales [..., dim / block], in 32 bits."""
    v = x.float().view(*x.shape[:-1], -1, block)
    top = v.abs().amax(dim=-1, keepdim=True)
    alive = top >= 127.0 * 2.0 ** -126
    scale = torch.where(alive, top / 127.0, 0.0)
    inverse = torch.where(alive, 127.0 / torch.where(alive, top, 1.0), 0.0)
    codes = torch.round(v * inverse).to(torch.int8)
    return codes.view(x.shape), scale.squeeze(-1)


def _put(cache, slots, k, v):
    """Writes tokens [T, heads, dim] into their slots."""
    kc, ks, vc, vs = cache
    page = kc.shape[2]
    block = kc.shape[3] // ks.shape[2]
    p, o = slots // page, slots % page
    codes, scales = _int8_blocks(k, block)
    kc[p, :, o] = codes
    ks[p, :, :, o] = scales
    codes, scales = _int8_blocks(v, block)
    vc[p, :, o // 16, :, o % 16] = codes
    vs[p, :, :, o] = scales


def _get(cache, pages, count):
    """The first `count` tokens of a sequence's pages as codes [count, heads, dim] and scales [count, heads, blocks]."""
    kc, ks, vc, vs = (t[pages] for t in cache)
    heads, dim = kc.shape[1], kc.shape[3]
    flat = lambda s: s.permute(0, 3, 1, 2).reshape(-1, heads, s.shape[2])[:count]
    return (kc.permute(0, 2, 1, 3).reshape(-1, heads, dim)[:count], flat(ks),
            vc.permute(0, 2, 4, 1, 3).reshape(-1, heads, dim)[:count], flat(vs))


def _empty_cache(case, pages):
    heads, dim, block, page = case["heads"], case["dim"], case["block"], case["page"]
    make = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device="cuda")
    return (make(pages, heads, page, dim, dtype=torch.int8), make(pages, heads, dim // block, page, dtype=torch.float32),
            make(pages, heads, page // 16, dim, 16, dtype=torch.int8),
            make(pages, heads, dim // block, page, dtype=torch.float32))


def _starts(counts):
    return torch.tensor([0] + counts, dtype=torch.int32).cumsum(0, dtype=torch.int32)


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    st = dict(op=op, case=case)
    if op == "mx4":
        st["x"] = _activations(g, case["rows"], case["cols"], case["gap"], case["dist"])
    elif op in ("linear", "product"):
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _activations(g, M, K, 0, case["dist"])
        st["w"] = _pack(_randn(g, N, K) * K ** -0.5)
        if op == "product":
            st["x"] = _pack(st["x"].float())
    else:
        lengths = _lengths(case)
        table, pages = _page_table(lengths, case["page"], seed)
        heads, dim, new = case["heads"], case["dim"], case["new"]
        cache = _empty_cache(case, pages)
        news = new if op == "cache" else 0                       # written by the pass itself
        for b, n in enumerate(lengths):
            for at in range(0, n - news, 16384):
                count = min(16384, n - news - at)
                k = _randn(g, count, heads, dim) * torch.exp(0.5 * _randn(g, 1, heads, 1))
                v = _randn(g, count, heads, dim)
                _put(cache, _slots(table, case["page"], b, at, count).cuda(), k.to(torch.bfloat16), v.to(torch.bfloat16))
        st.update(cache=cache, lengths=lengths, table=table.cuda())
        if op == "cache":
            rows = case["seqs"] * new                            # keys and values as a fused projection leaves them
            qkv = _randn(g, rows, 2 * heads * dim).to(torch.bfloat16)
            st["k"], st["v"] = qkv[:, :heads * dim].view(rows, heads, dim), qkv[:, heads * dim:].view(rows, heads, dim)
            st["slots"] = torch.cat([_slots(table, case["page"], b, n - new, new) for b, n in enumerate(lengths)]).cuda()
        else:
            st["q"] = _randn(g, case["seqs"] * new, heads * case["group"], dim).to(torch.bfloat16)
            st["scale"] = dim ** -0.5
    if own:
        _prepare_own(st, case)
    return st


def _prepare_own(st, case):
    """The plan of a program that uses the library: output buffers, workspaces, lengths and tables on the device."""
    from paper_2506_17615_amd import binding as eq
    empty = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    if case["op"] == "mx4":
        st["packed"] = eq.alloc_mx4(case["rows"], case["cols"])
        st["out"] = empty(case["rows"], case["cols"])
        return
    if case["op"] in ("linear", "product"):
        st["out"] = empty(case["M"], case["N"])
        st["workspace"] = eq.alloc_mx4_workspace(case["M"], case["N"], case["K"])
        return
    st["cache"] = eq.Cache(*st["cache"])
    st["device_lengths"] = torch.tensor(st["lengths"], dtype=torch.int32, device="cuda")
    if case["op"] == "cache":
        total = sum(st["lengths"])
        st["starts"] = _starts(st["lengths"]).cuda()
        st["out"] = empty(total, case["heads"], case["dim"]), empty(total, case["heads"], case["dim"])
    else:
        st["starts"] = _starts([case["new"]] * case["seqs"]).cuda()
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        st["workspace"] = eq.alloc_cache_attention_workspace(st["cache"], st["q"].shape[0], st["q"].shape[1], case["seqs"],
                                                             case["new"], case["longest"])


# ---------------------------------------------------------------- one pass

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2506_17615_amd import binding as eq
    op = st["op"]
    if op == "mx4":
        eq.equarx_mx4_quantize(st["x"], *st["packed"])
        eq.equarx_mx4_dequantize(*st["packed"], st["out"])
        return st["out"]
    if op == "linear":
        eq.equarx_mx4_linear(st["x"], *st["w"], st["out"], st["workspace"])
        return st["out"]
    if op == "product":
        eq.equarx_mx4_product(*st["x"], *st["w"], st["case"]["K"], st["out"], st["workspace"])
        return st["out"]
    if op == "cache":
        eq.equarx_cache_write(st["cache"], st["k"], st["v"], st["slots"])
        eq.equarx_cache_read(st["cache"], st["table"], st["device_lengths"], st["starts"], *st["out"])
        return st["out"]
    case = st["case"]
    eq.equarx_cache_attention(st["cache"], st["q"], st["starts"], st["table"], st["device_lengths"], st["out"], st["scale"],
                              case["new"], case["longest"], True, case["window"], st["lse"], st["workspace"])
    return st["out"], st["lse"]


def _rounded(x):
    """A tensor of rows as the values that its packed form stands for, fp32."""
    rows, cols = x.shape
    padded = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float32, device=x.device)
    padded[:, :cols] = x
    v = padded.view(rows, -1, 32)
    s = _shared_exponent(v)
    a = torch.ldexp(v, -s)
    m = a.abs()
    fine = torch.where(m < 2, torch.round(m * 2) / 2, torch.where(m < 4, torch.round(m), torch.round(m / 2) * 2))
    return torch.ldexp(torch.copysign(fine.clamp(max=6.0), a), s).view(rows, -1)[:, :cols]


def _run_plain(st):
    op, case = st["op"], st["case"]
    if op == "mx4":
        return _rounded(st["x"].float()).to(torch.bfloat16)
    if op in ("linear", "product"):
        x = _rounded(st["x"].float()) if op == "linear" else _unpack(*st["x"], case["K"])
        return torch.matmul(x, _unpack(*st["w"], case["K"]).t()).to(torch.bfloat16)
    lengths, table, cache = st["lengths"], st["table"], st["cache"]
    page, heads, dim = case["page"], case["heads"], case["dim"]
    wide = lambda codes, scales: codes.float() * scales.repeat_interleave(case["block"], dim=-1)
    if op == "cache":
        _put(cache, st["slots"], st["k"], st["v"])
        ks, vs = [], []
        for b, n in enumerate(lengths):
            kc, ksc, vc, vsc = _get(cache, table[b, :-(-n // page)].long(), n)
            ks.append(wide(kc, ksc).to(torch.bfloat16))
            vs.append(wide(vc, vsc).to(torch.bfloat16))
        return torch.cat(ks), torch.cat(vs)
    new, group, window = case["new"], case["group"], case["window"]
    outs, lses = [], []
    for b, n in enumerate(lengths):
        kc, ksc, vc, vsc = _get(cache, table[b, :-(-n // page)].long(), n)
        k, v = wide(kc, ksc).permute(1, 2, 0).contiguous(), wide(vc, vsc).permute(1, 0, 2).contiguous()
        q = st["q"][b * new:(b + 1) * new].float().view(new, heads, group, dim)
        q = q.permute(1, 2, 0, 3).reshape(heads, group * new, dim)
        at = torch.arange(n - new, n, device="cuda").unsqueeze(1)
        seen = torch.arange(n, device="cuda").unsqueeze(0)
        hidden = (seen > at) | (seen <= at - window) if window else seen > at
        s = (torch.bmm(q, k) * st["scale"]).view(heads, group, new, n).masked_fill_(hidden, -math.inf)
        top = s.amax(dim=-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(dim=-1, keepdim=True)
        o = torch.bmm(p.view(heads, group * new, n), v).view(heads, group, new, dim) / total
        outs.append(o.permute(2, 0, 1, 3).reshape(new, heads * group, dim).to(torch.bfloat16))
        lses.append((top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(new, heads * group))
    return torch.cat(outs), torch.cat(lses)


# ---------------------------------------------------------------- the definitions in 64 bits

def _nearest_mx4(x):
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


def _stands_for(codes, scales, cols):
    low, high = codes.to(torch.int16) % 16, codes.to(torch.int16) // 16
    nibble = torch.stack((low, high), dim=2).flatten(1)
    exponent, mantissa = (nibble % 8 // 2).double(), (nibble % 2).double()
    size = torch.where(exponent > 0, torch.exp2(exponent - 1) * (1 + mantissa / 2), mantissa / 2)
    size = torch.where(nibble >= 8, -size, size)
    return (size * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1))[:, :cols]


def exact(case, seed):
    with_own = own
    globals()["own"] = False
    try:
        st = prepare(case, seed)
    finally:
        globals()["own"] = with_own
    op = case["op"]
    if op == "mx4":
        return _nearest_mx4(st["x"].double())
    if op in ("linear", "product"):
        x = _nearest_mx4(st["x"].double()) if op == "linear" else _stands_for(*st["x"], case["K"])
        return x @ _stands_for(*st["w"], case["K"]).T
    page, heads, dim, block, new = case["page"], case["heads"], case["dim"], case["block"], case["new"]
    kc, ks, vc, vs = st["cache"]
    lengths = st["lengths"]

    def one(b, h, t):
        """Keys and values of sequence b's first t tokens in head h, from the codes, one scale per block."""
        p = st["table"][b, :(t + page - 1) // page].long()
        k = kc[p, h].double().reshape(-1, dim // block, block) * ks[p, h].double().transpose(1, 2).reshape(-1, dim // block, 1)
        v = vc[p, h].double().transpose(2, 3).reshape(-1, dim // block, block)
        v = v * vs[p, h].double().transpose(1, 2).reshape(-1, dim // block, 1)
        return k.reshape(-1, dim)[:t], v.reshape(-1, dim)[:t]

    def kept(x):
        """New tokens as the cache holds them: nearest multiple of a block's largest magnitude / 127."""
        w = x.double().reshape(*x.shape[:2], dim // block, block)
        top = w.abs().max(dim=-1, keepdim=True).values
        unit = (top / 127).clamp(min=1e-300)
        return (torch.round(w / unit) * unit).reshape(x.shape)

    if op == "cache":
        ks_out, vs_out = [], []
        for b, n in enumerate(lengths):
            pairs = [one(b, h, n) for h in range(heads)]
            k, v = (torch.stack([p[i] for p in pairs], dim=1) for i in (0, 1))
            k[n - new:], v[n - new:] = kept(st["k"][b * new:(b + 1) * new]), kept(st["v"][b * new:(b + 1) * new])
            ks_out.append(k)
            vs_out.append(v)
        return torch.cat(ks_out), torch.cat(vs_out)
    group, window = case["group"], case["window"]
    out = torch.zeros((len(lengths) * new, heads * group, dim), dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        rank = torch.arange(n, device="cuda")
        place = rank[n - new:, None]
        visible = rank[None, :] <= place
        if window:
            visible &= rank[None, :] > place - window
        for h in range(heads):
            k, v = one(b, h, n)
            for i in range(group):
                row = h * group + i
                logits = st["q"][b * new:(b + 1) * new, row].double() @ k.T * st["scale"]
                logits = torch.where(visible, logits, -math.inf)
                norm = torch.logsumexp(logits, dim=1)
                out[b * new:(b + 1) * new, row] = torch.exp(logits - norm[:, None]) @ v
                lse[b * new:(b + 1) * new, row] = norm
    return out, lse


# ---------------------------------------------------------------- what a pass cannot do without

def _pairs(n, new, window):
    """Query-key pairs of `new` queries at the end of n tokens."""
    return sum(min(p + 1, window) if window else p + 1 for p in range(n - new, n))


def work(case):
    """Inputs read once, outputs written once.  Quantizing and reading back count as the two operators they are: the packed
    form is one's output and the other's input.  Operations: a multiply-add is two; of a quantized element |.|, max,
    multiply and round, and a multiply to read it."""
    op = case["op"]
    if op == "mx4":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * (2 + 17 / 32), "flops": 5 * n}
    if op in ("linear", "product"):
        M, N, K = case["M"], case["N"], case["K"]
        x = 2 * M * K if op == "linear" else M * K * 17 / 32
        return {"bytes": x + N * K * 17 / 32 + 2 * M * N, "flops": 2 * M * N * K}
    heads, dim, block, new = case["heads"], case["dim"], case["block"], case["new"]
    lengths = _lengths(case)
    token = 2 * heads * dim * (1 + 4 / block)                    # keys and values of one token in the cache
    if op == "cache":
        written, read = case["seqs"] * new, sum(lengths)
        return {"bytes": written * (4 * heads * dim + token) + read * (token + 4 * heads * dim),
                "flops": 2 * heads * dim * (4 * written + read)}
    window, q_heads = case["window"], heads * case["group"]
    seen = sum(min(n, new + window - 1) if window else n for n in lengths)
    pairs = sum(_pairs(n, new, window) for n in lengths)
    rows = case["seqs"] * new * q_heads
    return {"bytes": seen * token + rows * (4 * dim + 4), "flops": 4 * pairs * q_heads * dim}
