"""The attention layer of paper_2506_17615_amd/serving.py: each of its stages against 64-bit arithmetic on what the stage before it
left, prompts first, then single tokens from a captured graph."""
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import serving

pytestmark = pytest.mark.gpu


def _values(packed, rows, cols):
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_dequantize(*packed, out)
    return out.double()


def _check_product(x, packed_w, n, got):
    """got against x (packed) times w: fp32 sums of K products, then a rounding to bf16."""
    rows, k = x.shape
    a, b = _values(serving.pack(x.contiguous()), rows, k), _values(packed_w, n, k)
    want, size = a @ b.T, a.abs() @ b.T.abs()
    assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (k + 8) * 2.0 ** -23 * size).all()


def _check(layer, x, starts, table, lengths, out, page):
    tokens, nq, nk = x.shape[0], layer.heads * layer.dim, layer.kv_heads * layer.dim
    for p in range(layer.shards):
        qkv, attended = layer.qkv[p, :tokens], layer.attended[p, :tokens]
        _check_product(x, layer.w_qkv[p], qkv.shape[1], qkv)
        cache = layer.caches[p]
        r = ref.CacheRef(cache.k_codes.shape[0], layer.kv_heads, page, layer.dim, 64)
        kc, ks, vc, vs = (t.cpu() for t in cache)
        r.codes = [kc.permute(0, 2, 1, 3).reshape(r.codes[0].shape), vc.permute(0, 2, 4, 1, 3).reshape(r.codes[1].shape)]
        r.scales = [t.permute(0, 3, 1, 2).reshape(r.scales[0].shape) for t in (ks, vs)]
        q = qkv[:, :nq].reshape(tokens, layer.heads, layer.dim).double().cpu()
        for b, n in enumerate(lengths):
            rows = slice(starts[b], starts[b + 1])
            want, _, mass, size = ref.attention(r, q[rows], table[b].tolist(), n, layer.dim ** -0.5, True, 0)
            e = (layer.dim + 8) * 2.0 ** -23 * size + 2.0 ** -20 + (n + 64) * 2.0 ** -23
            bound = 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2.02 * e[..., None]) * mass
            assert ((attended[rows].double().cpu() - want).abs() <= bound).all(), (p, b)
        _check_product(attended.flatten(1), layer.w_o[p], layer.hidden, layer.partials[p, :tokens])
    parts = [layer.partials[p, :tokens].reshape(-1) for p in range(layer.shards)]
    want = torch.empty_like(out)
    eq.equarx_reduce_quantized(parts, layer.wire_block, want.view(-1), eq.alloc_workspace(layer.shards, out.numel(), layer.wire_block))
    assert torch.equal(out, want)


@pytest.mark.parametrize("shards,heads,kv_heads,dim", ((2, 8, 4, 64), (4, 8, 8, 128)))
def test_prompts_then_single_tokens(shards, heads, kv_heads, dim):
    hidden, page, prompts, steps = 320, 16, [19, 33, 1], 3
    gen = torch.Generator().manual_seed(7)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).mul_(shape[-1] ** -0.5).to(torch.bfloat16).cuda()
    width = 3
    table = torch.randperm(3 * width, generator=gen).to(torch.int32).view(3, width)
    layer = serving.ShardedAttention(bf16((heads + 2 * kv_heads) * dim, hidden), bf16(hidden, heads * dim), shards, heads, kv_heads, dim,
                                     3 * width, page, sum(prompts), 3, 40)
    x, out = bf16(sum(prompts), hidden) * 10, torch.empty(sum(prompts), hidden, dtype=torch.bfloat16, device="cuda")
    starts = [0, 19, 52, 53]
    device_table, lengths = table.cuda(), torch.tensor(prompts, dtype=torch.int32).cuda()
    layer(x, serving.slots_of(table, page, prompts, prompts).cuda(), torch.tensor(starts, dtype=torch.int32).cuda(), device_table, lengths, 33, out)
    _check(layer, x, starts, table, prompts, out, page)

    token, step_out, slots = torch.empty_like(x[:3]), torch.empty_like(out[:3]), torch.empty(3, dtype=torch.int64, device="cuda")
    one = torch.arange(4, dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(token, slots, one, device_table, lengths, 1, step_out)
    for step in range(steps):
        now = [n + step + 1 for n in prompts]
        token.copy_(x[5 * step:5 * step + 3])
        lengths.copy_(torch.tensor(now))
        slots.copy_(serving.slots_of(table, page, now, [1] * 3))
        graph.replay()
        torch.cuda.synchronize()
        _check(layer, token, [0, 1, 2, 3], table, now, step_out, page)


def test_what_a_layer_refuses():
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        serving.ShardedAttention(w, w, 3, 8, 4, 64, 4, 16, 8, 1, 64)
    with pytest.raises(ValueError):
        serving.ShardedAttention(w, w, 1, 8, 4, 64, 4, 16, 8, 1, 64)
