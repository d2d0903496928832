"""An attention layer of a tensor-parallel server on one device: the operators of the library in the order they are used in.

Shard p of P has 1/P of the heads.  It projects the new tokens with its 4-bit rows of the joint q, k, v weights, writes keys and
values into its int8 cache, attends over the cache, and projects its heads with its 4-bit columns of the output weights; the
P partial sums are then reduced as the all-reduce between the shards would be (`equarx_reduce_fused`).

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
        # one workspace serves every call in turn, of the largest size that any has
        sizes = [eq.alloc_cache_attention_workspace(self.caches[0], max_tokens, self.heads, sequences, None, max_length, device="meta")]
        sizes += [eq.alloc_mx4_workspace(max_tokens, r, k, device="meta") for r, k in ((rows, hidden), (hidden, self.heads * dim))]
        self.workspace = torch.empty(max(s.numel() for s in sizes), dtype=torch.uint8, device="cuda")

    def __call__(self, x, slots, q_starts, page_table, lengths, max_queries, out):
        """out bf16 [tokens, hidden] <- the layer for x bf16 [tokens, hidden], whose sequence b is q_starts[b] .. q_starts[b + 1] - 1
        and stands at the end of lengths[b] tokens, its own among them; slots: where its keys and values go."""
        tokens = x.shape[0]
        if not 1 <= tokens <= self.max_tokens:
            raise ValueError(f"x: need 1 to {self.max_tokens} tokens")
        nq, nk = self.heads * self.dim, self.kv_heads * self.dim
        max_queries = max(max_queries, -(-tokens // max(page_table.shape[0], 1)))      # no run can be shorter than the mean
        for p in range(self.shards):
            qkv, attended, cache = self.qkv[p, :tokens], self.attended[p, :tokens], self.caches[p]
            eq.equarx_mx4_linear(x, *self.w_qkv[p], qkv, self.workspace)
            q, k, v = (t.unflatten(1, (-1, self.dim)) for t in qkv.split([nq, nk, nk], dim=1))
            eq.equarx_cache_write(cache, k, v, slots)
            eq.equarx_cache_attention(cache, q, q_starts, page_table, lengths, attended, self.dim ** -0.5, max_queries, self.max_length,
                                      workspace=self.workspace)
            eq.equarx_mx4_linear(attended.flatten(1), *self.w_o[p], self.partials[p, :tokens], self.workspace)
        eq.equarx_reduce_fused([self.partials[p, :tokens].reshape(-1) for p in range(self.shards)], self.wire_block, out.view(-1))


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


def main():
    shards, heads, kv_heads, dim, hidden, page = 8, 32, 16, 128, 5376, 64
    prompts, steps = [700, 1500, 64, 1], 32
    longest = max(prompts) + steps
    gen = torch.Generator().manual_seed(0)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).mul_(shape[-1] ** -0.5).to(torch.bfloat16).cuda()
    width = -(-longest // page)
    table = torch.randperm(len(prompts) * width, generator=gen).to(torch.int32).view(len(prompts), width)
    layer = ShardedAttention(bf16((heads + 2 * kv_heads) * dim, hidden), bf16(hidden, heads * dim), shards, heads, kv_heads, dim,
                             table.numel(), page, sum(prompts), len(prompts), longest)
    on = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")
    x, out = bf16(sum(prompts), hidden), torch.empty(sum(prompts), hidden, dtype=torch.bfloat16, device="cuda")
    starts, device_table = on([0] + prompts).cumsum(0, dtype=torch.int32), table.cuda()
    prompt_slots, lengths = slots_of(table, page, prompts, prompts).cuda(), on(prompts)

    def timed(f, count=1):
        f()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(count):
            f()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / count * 1e3

    us = timed(lambda: layer(x, prompt_slots, starts, device_table, lengths, max(prompts), out))
    print(f"prompts of {prompts} tokens: {us:.0f} us, {sum(prompts) / us * 1e6:.0f} tokens/s a layer")
    # a decode step as a graph: the device holds the lengths and slots, and moves them on itself
    token, step_out = x[:len(prompts)].clone(), out[:len(prompts)]
    one = on(list(range(len(prompts) + 1)))
    rows = torch.arange(len(prompts), device="cuda")

    def step():
        lengths.add_(1).clamp_(max=longest)
        last = (lengths - 1).long()
        slots = device_table[rows, last // page].long() * page + last % page
        layer(token, slots, one, device_table, lengths, 1, step_out)

    graph = captured(step)
    us = timed(graph.replay, steps - 2)
    print(f"decode of {len(prompts)} sequences: {us:.0f} us a step and layer")


if __name__ == "__main__":
    main()
