"""An attention layer of a tensor-parallel server on one device: the operators of the library in the order they are used in.

Shard p of P has 1/P of the heads.  It projects the new tokens with its 4-bit rows of the joint q, k, v weights, writes keys and
values into its int8 cache, attends over the cache, and projects its heads with its 4-bit columns of the output weights; the
P partial sums are then reduced as the all-reduce between the shards would be (`equarx_reduce_fused`), or reduced, added to the residual
stream and normed for the next layer in one launch (`equarx_norm_reduced`).  Requests may have low-rank adapters beside both projections.

    python -m paper_2506_17615_amd.serving            # prompts, then decode steps from a captured graph
"""
import torch

from . import binding as eq


def pack(weights: torch.Tensor):
    """Weights bf16 [rows, cols] in the 4-bit form: codes, scales."""
    packed = eq.alloc_mx4(*weights.shape, device=weights.device)
    eq.equarx_mx4_quantize(weights, *packed)
    return packed


class ShardedAttention:
    """Weights, caches and buffers of a layer for calls of up to max_tokens new tokens, of up to `sequences` sequences.

    w_qkv bf16 [(heads + 2 * kv_heads) * dim, hidden], heads of q before those of k and v; w_o bf16 [hidden, heads * dim].
    Its calls share the buffers and the workspace: they go to one stream, or to streams that wait for each other.
    """

    def __init__(self, w_qkv, w_o, shards, heads, kv_heads, dim, pages, page, max_tokens, sequences, max_length, block=64,
                 wire_block=256):
        hidden = w_o.shape[0]
        if heads % shards or kv_heads % shards or heads % kv_heads:
            raise ValueError("heads: need a multiple of kv_heads, and both multiples of shards")
        if tuple(w_qkv.shape) != ((heads + 2 * kv_heads) * dim, hidden) or w_o.shape[1] != heads * dim:
            raise ValueError("w_qkv, w_o: need [(heads + 2 * kv_heads) * dim, hidden] and [hidden, heads * dim]")
        self.shards, self.heads, self.kv_heads, self.dim, self.hidden = shards, heads // shards, kv_heads // shards, dim, hidden
        self.max_tokens, self.max_length, self.wire_block = max_tokens, max_length, wire_block
        q, k, v = w_qkv.split([heads * dim, kv_heads * dim, kv_heads * dim])
        parts = zip(q.chunk(shards), k.chunk(shards), v.chunk(shards))
        self.w_qkv = [pack(torch.cat(p)) for p in parts]
        self.w_o = [pack(p) for p in w_o.chunk(shards, dim=1)]
        self.caches = [eq.alloc_cache(pages, self.kv_heads, page, dim, block) for _ in range(shards)]
        rows = (self.heads + 2 * self.kv_heads) * dim
        new = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        self.qkv, self.attended = new(shards, max_tokens, rows), new(shards, max_tokens, self.heads, dim)
        self.partials = new(shards, max_tokens, hidden)
        self.adapters = None
        # one workspace serves every call in turn, of the largest size that any has
        sizes = [eq.alloc_cache_attention_workspace(self.caches[0], max_tokens, self.heads, sequences, None, max_length, device="meta")]
        sizes += [eq.alloc_mx4_workspace(max_tokens, r, k, device="meta") for r, k in ((rows, hidden), (hidden, self.heads * dim))]
        self.workspace = torch.empty(max(s.numel() for s in sizes), dtype=torch.uint8, device="cuda")

    def add_adapters(self, a_qkv, b_qkv, a_o, b_o, factors):
        """Low-rank adapters beside the projections: a_qkv bf16 [adapters, 3 * rank, hidden] (of q, k and v), b_qkv [adapters, (heads + 2 * kv_heads)
        * dim, rank], a_o [adapters, rank, heads * dim], b_o [adapters, hidden, rank], factors fp32 [adapters]."""
        adapters, rank, shards, dim = b_o.shape[0], b_o.shape[2], self.shards, self.dim
        rows = (self.heads + 2 * self.kv_heads) * dim
        if (tuple(a_qkv.shape) != (adapters, 3 * rank, self.hidden) or tuple(b_qkv.shape) != (adapters, shards * rows, rank)
                or tuple(a_o.shape) != (adapters, rank, shards * self.heads * dim) or b_o.shape[1] != self.hidden or factors.numel() != adapters):
            raise ValueError("adapters: need a_qkv [n, 3 * rank, hidden], b_qkv [n, (heads + 2 * kv_heads) * dim, rank], a_o [n, rank, heads * dim], "
                             "b_o [n, hidden, rank], factors [n]")
        nq, nk = self.heads * dim, self.kv_heads * dim
        parts = zip(*(t.chunk(shards, dim=1) for t in b_qkv.split([shards * nq, shards * nk, shards * nk], dim=1)))
        sizes = ((self.max_tokens, rows, self.hidden, rank, 3, adapters), (self.max_tokens, self.hidden, nq, rank, 1, adapters))
        sizes = [eq.alloc_adapters_workspace(*z, device="meta").numel() for z in sizes]
        self.adapters = dict(a_qkv=a_qkv.contiguous(), b_qkv=[torch.cat(p, dim=1) for p in parts], b_o=b_o.contiguous(), factors=factors,
                             a_o=[p.contiguous() for p in a_o.chunk(shards, dim=2)], ends=(nq, nq + nk, rows),
                             workspace=torch.empty(max(sizes), dtype=torch.uint8, device="cuda"))

    def _project(self, x, slots, q_starts, page_table, lengths, max_queries, ids):
        """The shards' partial sums for x; ids int32 [tokens]: every token's adapter, None or an entry outside the adapters' for none."""
        tokens = x.shape[0]
        if not 1 <= tokens <= self.max_tokens:
            raise ValueError(f"x: need 1 to {self.max_tokens} tokens")
        if ids is not None and self.adapters is None:
            raise ValueError("ids: there are no adapters")
        nq, nk, more = self.heads * self.dim, self.kv_heads * self.dim, self.adapters
        max_queries = max(max_queries, -(-tokens // max(page_table.shape[0], 1)))      # no run can be shorter than the mean
        # attention leaves rows of no sequence as they are: they would be another step's, or what the memory held
        self.attended[:, :tokens].zero_()
        for p in range(self.shards):
            qkv, attended, cache, partial = self.qkv[p, :tokens], self.attended[p, :tokens], self.caches[p], self.partials[p, :tokens]
            eq.equarx_mx4_linear(x, *self.w_qkv[p], qkv, self.workspace)
            if ids is not None:
                eq.equarx_adapters(x, more["a_qkv"], more["b_qkv"][p], more["factors"], ids, qkv, more["ends"], more["workspace"])
            q, k, v = (t.unflatten(1, (-1, self.dim)) for t in qkv.split([nq, nk, nk], dim=1))
            eq.equarx_cache_write(cache, k, v, slots)
            eq.equarx_cache_attention(cache, q, q_starts, page_table, lengths, attended, self.dim ** -0.5, max_queries, self.max_length,
                                      workspace=self.workspace)
            eq.equarx_mx4_linear(attended.flatten(1), *self.w_o[p], partial, self.workspace)
            if ids is not None:
                eq.equarx_adapters(attended.flatten(1), more["a_o"][p], more["b_o"], more["factors"], ids, partial, None, more["workspace"])

    def __call__(self, x, slots, q_starts, page_table, lengths, max_queries, out, ids=None):
        """out bf16 [tokens, hidden] <- the layer for x bf16 [tokens, hidden], whose sequence b is q_starts[b] .. q_starts[b + 1] - 1
        and stands at the end of lengths[b] tokens, its own among them; slots: where its keys and values go.  Rows of no sequence
        become zeros."""
        self._project(x, slots, q_starts, page_table, lengths, max_queries, ids)
        tokens = x.shape[0]
        eq.equarx_reduce_fused([self.partials[p, :tokens].reshape(-1) for p in range(self.shards)], self.wire_block, out.view(-1))

    def normed(self, x, slots, q_starts, page_table, lengths, max_queries, residual, weight, out, eps=1e-6, ids=None):
        """The layer for normed rows x: residual <- residual + what __call__ writes, out <- its norm times weight, the next layer's x.
        Residual rows of no sequence stay as they are."""
        self._project(x, slots, q_starts, page_table, lengths, max_queries, ids)
        tokens = x.shape[0]
        eq.equarx_norm_reduced([self.partials[p, :tokens] for p in range(self.shards)], self.wire_block, weight, eps, residual, out)


def slots_of(page_table, page, lengths, new):
    """int64: where the last new[b] of the lengths[b] tokens of every sequence are."""
    rows = []
    for b, (n, count) in enumerate(zip(lengths, new)):
        t = torch.arange(n - count, n)
        rows.append(page_table[b, t // page].long() * page + t % page)
    return torch.cat(rows)


def captured(step):
    """A graph of step: run once on a stream of its own, after what the current one has been given, then captured."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    return graph


class Requests:
    """Sequences in places of a page table on the device: what a step of them reads, made there by one launch or two.

    rows: of a step, at most.  A step's q_starts, slots and row_tags are those of its first `rows` rows, counts[b] of sequence b after those of the
    sequences before it.  Rows behind the last sequence, and of one that got none of the tokens it wanted (granted[b] is 0: no pages are
    left, or no room), have slot -1 and tag -1: nothing is kept in the cache for them, no adapter is theirs, and the layer adds nothing to them."""

    def __init__(self, sequences, width, pages, page, rows):
        self.page, self.pages = page, eq.alloc_pages(sequences, width, pages)
        ints = lambda n, dtype=torch.int32: torch.zeros(n, dtype=dtype, device="cuda")
        self.q_starts, self.granted, self.seen, self.tags = ints(sequences + 1), ints(sequences), ints(sequences), ints(sequences) - 1
        self.slots, self.row_tags = ints(rows, torch.int64), ints(rows)

    def step(self, counts, rows):
        """counts int32 [sequences] more tokens for every sequence, up to `rows` in all: all that it wants, or none."""
        eq.equarx_pages_extend(self.pages, self.page, counts, self.q_starts, self.slots[:rows], self.granted, None, self.tags, self.row_tags[:rows],
                               self.seen)
        return dict(slots=self.slots[:rows], q_starts=self.q_starts, page_table=self.pages.table, lengths=self.seen), self.row_tags[:rows]

    def keep(self, tokens):
        """Takes every sequence back to its first tokens[b] (0: it has ended)."""
        eq.equarx_pages_trim(self.pages, self.page, tokens)


def main():
    shards, heads, kv_heads, dim, hidden, page, rank, adapters = 8, 32, 16, 128, 5376, 64, 16, 4
    prompts, steps = [700, 1500, 64, 1], 32
    longest = max(prompts) + steps
    gen = torch.Generator().manual_seed(0)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).mul_(shape[-1] ** -0.5).to(torch.bfloat16).cuda()
    width, rows = -(-longest // page), (heads + 2 * kv_heads) * dim
    layer = ShardedAttention(bf16(rows, hidden), bf16(hidden, heads * dim), shards, heads, kv_heads, dim, len(prompts) * width, page, sum(prompts),
                             len(prompts), longest)
    layer.add_adapters(bf16(adapters, 3 * rank, hidden), bf16(adapters, rows, rank), bf16(adapters, rank, heads * dim), bf16(adapters, hidden, rank),
                       torch.full((adapters,), 0.5, device="cuda"))
    on = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")
    requests = Requests(len(prompts), width, len(prompts) * width, page, sum(prompts))
    requests.tags.copy_(on([2, -1, 0, 2]))                                 # one request without an adapter
    stream, weight, nothing = bf16(sum(prompts), hidden), 1 + bf16(hidden), on([0] * len(prompts))
    x, out = torch.empty_like(stream), torch.empty_like(stream)
    counts = on(prompts)

    def timed(f, count=1):
        f()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(count):
            f()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / count * 1e3

    def prompt():
        requests.keep(nothing)
        step, ids = requests.step(counts, sum(prompts))
        eq.equarx_norm(stream, weight, out=x)
        layer.normed(x, **step, max_queries=max(prompts), residual=stream, weight=weight, out=out, ids=ids)

    us = timed(prompt)
    print(f"prompts of {prompts} tokens: {us:.0f} us, {sum(prompts) / us * 1e6:.0f} tokens/s a layer")
    # a decode step as a graph: the device hands out slots and pages and moves the lengths on itself
    token, token_x, token_out, one = (t[:len(prompts)] for t in (stream, x, out, on([1] * len(prompts))))

    def decode():
        step, ids = requests.step(one, len(prompts))
        eq.equarx_norm(token, weight, out=token_x)
        layer.normed(token_x, **step, max_queries=1, residual=token, weight=weight, out=token_out, ids=ids)

    graph = captured(decode)
    us = timed(graph.replay, steps - 2)
    print(f"decode of {len(prompts)} sequences: {us:.0f} us a step and layer")


if __name__ == "__main__":
    main()
