"""Norms, adapters and page tables together, as the serving layer uses them: requests of several adapters enter, go on from a captured graph, are taken
back a few tokens, end and make room.  Every stage is held to 64-bit arithmetic, or to the calls it is made of, on what the stage before left."""
import pytest
import torch

import test_adapters_gpu as lora
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import serving

pytestmark = pytest.mark.gpu

SHARDS, HEADS, KV, DIM, HIDDEN, PAGE, RANK, ADAPTERS = 2, 8, 4, 64, 384, 16, 8, 3


def _layer(max_tokens, sequences, pages, longest):
    gen = torch.Generator().manual_seed(3)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).mul_(shape[-1] ** -0.5).to(torch.bfloat16).cuda()
    rows = (HEADS + 2 * KV) * DIM
    layer = serving.ShardedAttention(bf16(rows, HIDDEN), bf16(HIDDEN, HEADS * DIM), SHARDS, HEADS, KV, DIM, pages, PAGE, max_tokens, sequences, longest,
                                     wire_block=128)
    whole = dict(a_qkv=bf16(ADAPTERS, 3 * RANK, HIDDEN), b_qkv=bf16(ADAPTERS, rows, RANK), a_o=bf16(ADAPTERS, RANK, HEADS * DIM),
                 b_o=bf16(ADAPTERS, HIDDEN, RANK), factors=torch.tensor([0.5, -2.0, 1.0]).cuda())
    layer.add_adapters(*whole.values())
    return layer, whole, bf16


def _shard_b(whole, p):
    """The rows of b_qkv that are shard p's heads, one by one."""
    nq, nk = HEADS * DIM, KV * DIM
    rows = []
    for start, n in ((0, nq), (nq, nk), (nq + nk, nk)):
        rows += range(start + p * n // SHARDS, start + (p + 1) * n // SHARDS)
    return whole["b_qkv"][:, rows]


def _check_step(layer, whole, x, ids, tokens):
    """The shards' projections with the adapters, from what the layer's buffers hold."""
    nq, nk = layer.heads * DIM, layer.kv_heads * DIM
    plain = torch.empty_like(layer.qkv[0, :tokens])
    for p in range(SHARDS):
        eq.equarx_mx4_linear(x, *layer.w_qkv[p], plain, layer.workspace)
        case = dict(x=x, a=whole["a_qkv"], b=_shard_b(whole, p), factors=whole["factors"], ids=ids, out=plain, widths=(nq, nk, nk))
        lora._check(case, layer.qkv[p, :tokens], "cuda")
        attended = layer.attended[p, :tokens].flatten(1)
        partial = torch.empty_like(layer.partials[p, :tokens])
        eq.equarx_mx4_linear(attended, *layer.w_o[p], partial, layer.workspace)
        case = dict(x=attended, a=whole["a_o"].chunk(SHARDS, dim=2)[p], b=whole["b_o"], factors=whole["factors"], ids=ids, out=partial, widths=(HIDDEN,))
        lora._check(case, layer.partials[p, :tokens], "cuda")


def _check_norm(layer, before, residual, weight, out, tokens):
    parts = [layer.partials[p, :tokens].reshape(-1) for p in range(SHARDS)]
    reduced, want, stream = torch.empty_like(out), torch.empty_like(out), before.clone()
    eq.equarx_reduce_fused(parts, layer.wire_block, reduced.view(-1))
    eq.equarx_norm(reduced, weight, residual=stream, out=want)
    assert torch.equal(residual, stream) and torch.equal(out, want)


def test_requests_come_go_on_and_end():
    sequences, rows, width = 4, 64, 6
    layer, whole, bf16 = _layer(rows, sequences, 16, width * PAGE)
    requests = serving.Requests(sequences, width, 16, PAGE, rows)
    on = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    requests.tags.copy_(on([2, 0, -1, 2]))
    weight, stream = 1 + bf16(HIDDEN), 3 * bf16(rows, HIDDEN)
    x, out = torch.empty_like(stream), torch.empty_like(stream)

    def run(counts, tokens, max_queries):
        step, ids = requests.step(counts, tokens)
        eq.equarx_norm(stream[:tokens], weight, out=x[:tokens])
        layer.normed(x[:tokens], **step, max_queries=max_queries, residual=stream[:tokens], weight=weight, out=out[:tokens], ids=ids)

    def check(lengths, counts, tokens, before):
        torch.cuda.synchronize()
        assert requests.pages.lengths.tolist() == lengths
        real = sum(counts)
        assert requests.q_starts.tolist() == [sum(counts[:b]) for b in range(sequences + 1)]
        want = serving.slots_of(requests.pages.table.cpu(), PAGE, lengths, counts)
        assert torch.equal(requests.slots[:real].cpu(), want) and (requests.slots[real:tokens] == -1).all()
        assert requests.row_tags[:tokens].tolist() == [t for b, t in enumerate([2, 0, -1, 2]) for _ in range(counts[b])] + [-1] * (tokens - real)
        _check_step(layer, whole, x[:tokens], requests.row_tags[:tokens], tokens)
        _check_norm(layer, before, stream[:tokens], weight, out[:tokens], tokens)

    # prompts, with rows to spare
    layer.attended.zero_()
    before = stream.clone()
    run(on([19, 33, 0, 5]), rows, 33)
    check([19, 33, 0, 5], [19, 33, 0, 5], rows, before)

    # single tokens from a graph, whose third sequence begins with its own first token
    one = on([1, 1, 1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(one, 4, 1)
    lengths = [19, 33, 0, 5]
    for _ in range(3):
        before = stream[:4].clone()
        graph.replay()
        lengths = [n + 1 for n in lengths]
        check(lengths, [1] * 4, 4, before)

    # two tokens back for the first, the second has ended and another takes its place, in eager calls between two replays
    requests.keep(on([20, 0, 100, 100]))
    lengths = [20, 0, lengths[2], lengths[3]]
    before = stream[:30].clone()
    run(on([0, 30, 0, 0]), 30, 30)
    lengths[1] = 30
    check(lengths, [0, 30, 0, 0], 30, before)
    before = stream[:4].clone()
    graph.replay()
    lengths = [n + 1 for n in lengths]
    check(lengths, [1] * 4, 4, before)
    held = [e for b, n in enumerate(lengths) for e in requests.pages.table[b, :-(-n // PAGE)].tolist()]
    assert sorted(held + requests.pages.free[:int(requests.pages.free_count)].tolist()) == list(range(16))


def test_a_layer_without_adapters_has_none():
    layer, whole, bf16 = _layer(8, 2, 4, 32)
    x, out = bf16(4, HIDDEN), torch.empty(4, HIDDEN, dtype=torch.bfloat16, device="cuda")
    requests = serving.Requests(2, 2, 4, PAGE, 8)
    step, ids = requests.step(torch.tensor([3, 1], dtype=torch.int32, device="cuda"), 4)
    layer(x, **step, max_queries=3, out=out)
    plain = out.clone()
    layer(x, **step, max_queries=3, out=out, ids=ids)                       # every tag is -1
    assert torch.equal(out, plain)
    layer.adapters = None
    with pytest.raises(ValueError):
        layer(x, **step, max_queries=3, out=out, ids=ids)
    with pytest.raises(ValueError):
        layer.add_adapters(*(t[:, :1] for t in list(whole.values())[:4]), whole["factors"])
