"""Rows of a step that are no sequence's: the serving layer adds nothing for them, whatever its buffers and the rows hold."""
import pytest
import torch

import serving_ref as ref
import test_serving_requests_gpu as layers
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import serving

pytestmark = pytest.mark.gpu

HIDDEN, PAGE = layers.HIDDEN, layers.PAGE


def _on(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("ids", (False, True))
def test_rows_behind_the_last_sequence_add_nothing(ids):
    rows, counts = 24, [5, 0, 9]
    real = sum(counts)
    layer, _, bf16 = layers._layer(rows, 3, 8, 2 * PAGE)
    requests = serving.Requests(3, 2, 8, PAGE, rows)
    requests.tags.copy_(_on([1, 0, 2]))
    weight, before = 1 + bf16(HIDDEN), 3 * bf16(rows, HIDDEN)
    x, out, stream = bf16(rows, HIDDEN), torch.empty_like(before), before.clone()
    x[real:] = float("nan")
    step, tags = requests.step(_on(counts), rows)
    if ids:
        tags[real:] = 1                                                 # a caller's own rows of adapters
    layer.attended.fill_(float("nan"))
    layer.normed(x, **step, max_queries=9, residual=stream, weight=weight, out=out, ids=tags if ids else None)
    assert torch.equal(stream[real:], before[real:]) and not torch.equal(stream[:real], before[:real])
    assert stream.isfinite().all() and out.isfinite().all()
    want = torch.empty_like(out)
    eq.equarx_norm(stream, weight, out=want)
    assert torch.equal(out, want)
    layer.attended.fill_(float("nan"))
    layer(x, **step, max_queries=9, out=out, ids=tags if ids else None)
    assert out[:real].isfinite().all() and not out[real:].any()


def test_a_graph_forgets_what_the_last_step_left():
    """A replay of a few rows after a step of many, whose rows hold other requests' attention."""
    rows = 24
    layer, _, bf16 = layers._layer(rows, 3, 12, 4 * PAGE)
    requests = serving.Requests(3, 4, 12, PAGE, rows)
    weight, stream = 1 + bf16(HIDDEN), 3 * bf16(rows, HIDDEN)
    x, out, counts = bf16(rows, HIDDEN), torch.empty_like(stream), _on([1, 0, 1])
    layer.normed(x, **requests.step(_on([8, 7, 9]), rows)[0], max_queries=9, residual=stream, weight=weight, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.normed(x[:8], **requests.step(counts, 8)[0], max_queries=1, residual=stream[:8], weight=weight, out=out[:8])
    for replay in range(4):
        if replay == 2:                                                 # a longer step between two replays
            layer.normed(x, **requests.step(_on([2, 9, 13]), rows)[0], max_queries=13, residual=stream, weight=weight, out=out)
        before = stream.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(stream[2:], before[2:]) and not torch.equal(stream[:2], before[:2])
        assert stream.isfinite().all() and out[:8].isfinite().all()


def _check_caches(layer, before, x, seqs):
    """The caches hold what they held, and in the tokens' slots the keys and values of the sequences' own rows: seqs has (row, count, slots)."""
    nq, nk = layer.heads * layer.dim, layer.kv_heads * layer.dim
    slots = torch.full((x.shape[0],), -1)
    for row, count, at in seqs:
        slots[row:row + count] = at
    for p, cache in enumerate(layer.caches):
        _, k, v = (t.unflatten(1, (-1, layer.dim)) for t in layer.qkv[p, :x.shape[0]].split([nq, nk, nk], dim=1))
        want = eq.Cache(*(t.clone() for t in before[p]))
        eq.equarx_cache_write(want, k, v, slots.cuda())
        assert all(torch.equal(a, b) for a, b in zip(want, cache))


def test_a_refused_sequence_moves_no_other():
    """A captured decode step whose pages run out: every sequence's row stays its own, with its own slot, adapter and attention, and the refused one's
    residual stays as it is."""
    sequences, pages, lengths = 4, 4, [5, 16, 3, 9]
    layer, whole, bf16 = layers._layer(40, sequences, pages, 3 * PAGE)
    requests = serving.Requests(sequences, 3, pages, PAGE, 40)
    tags = [2, 0, -1, 1]
    requests.tags.copy_(_on(tags))
    weight, stream = 1 + bf16(HIDDEN), 3 * bf16(40, HIDDEN)
    x, out = bf16(40, HIDDEN), torch.empty_like(stream)
    step, ids = requests.step(_on(lengths), 40)
    layer.normed(x, **step, max_queries=16, residual=stream, weight=weight, out=out, ids=ids)
    assert requests.granted.tolist() == lengths and not int(requests.pages.free_count)

    one = _on([1] * sequences)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step, ids = requests.step(one, sequences)
        layer.normed(x[:4], **step, max_queries=1, residual=stream[:4], weight=weight, out=out[:4], ids=ids)

    def replay(refused, bad):
        x.copy_(10 * bf16(40, HIDDEN))
        if bad:                                                         # what a row holds that nobody asks for
            x[refused] = float("nan")
        before, caches = stream.clone(), [[t.clone() for t in c] for c in layer.caches]
        graph.replay()
        torch.cuda.synchronize()
        served = [b for b in range(sequences) if b != refused]
        for b in served:
            lengths[b] += 1
        assert requests.granted.tolist() == [int(b != refused) for b in range(sequences)]
        assert requests.pages.lengths.tolist() == lengths and requests.q_starts.tolist() == [0, 1, 2, 3, 4]
        table = requests.pages.table.cpu()
        slot = [int(table[b, (lengths[b] - 1) // PAGE]) * PAGE + (lengths[b] - 1) % PAGE for b in range(sequences)]
        assert requests.slots[:4].tolist() == [-1 if b == refused else slot[b] for b in range(sequences)]
        assert requests.row_tags[:4].tolist() == [-1 if b == refused else tags[b] for b in range(sequences)]
        _check_caches(layer, caches, x[:4], [(b, 1, torch.tensor([slot[b]])) for b in served])
        assert not layer.attended[:, refused].any()
        assert torch.equal(stream[refused], before[refused]) and out[refused].isfinite().all()
        for p in range(layer.shards):
            _check_attention(layer, p, table, lengths, served)
        if not bad:
            layers._check_step(layer, whole, x[:4], requests.row_tags[:4], 4)
            layers._check_norm(layer, before[:4], stream[:4], weight, out[:4], 4)

    for bad in (False, True, False):
        replay(1, bad)                                                  # its seventeenth token would need a page
    requests.keep(_on([100, 100, 100, 0]))                              # the last one ends and begins anew: the second, before it, has its page
    lengths[3] = 0
    for bad in (True, False):
        replay(3, bad)


def _check_attention(layer, p, table, lengths, served):
    """The attended rows of the last step against 64-bit arithmetic over what the cache holds."""
    r = ref.CacheRef(layer.caches[p].k_codes.shape[0], layer.kv_heads, PAGE, layer.dim, 64)
    kc, ks, vc, vs = (t.cpu() for t in layer.caches[p])
    r.codes = [kc.permute(0, 2, 1, 3).reshape(r.codes[0].shape), vc.permute(0, 2, 4, 1, 3).reshape(r.codes[1].shape)]
    r.scales = [t.permute(0, 3, 1, 2).reshape(r.scales[0].shape) for t in (ks, vs)]
    for b in served:
        q = layer.qkv[p, b:b + 1, :layer.heads * layer.dim].reshape(1, layer.heads, layer.dim).double().cpu()
        want, _, mass, size = ref.attention(r, q, table[b].tolist(), lengths[b], layer.dim ** -0.5, True, 0)
        e = (layer.dim + 8) * 2.0 ** -23 * size + 2.0 ** -20 + (lengths[b] + 64) * 2.0 ** -23
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2.02 * e[..., None]) * mass
        assert ((layer.attended[p, b:b + 1].double().cpu() - want).abs() <= bound).all(), (p, b)


@pytest.mark.parametrize("long", (300, 40))
def test_prompts_that_get_nothing_keep_nothing(long):
    """One that the pages have no room for, and one that ends behind the last row."""
    layer, _, bf16 = layers._layer(400, 4, 4, 25 * PAGE)
    requests = serving.Requests(4, 25, 4, PAGE, 400)
    requests.tags.copy_(_on([1, 2, 0, 1]))
    weight, before = 1 + bf16(HIDDEN), 3 * bf16(400, HIDDEN)
    x, out, stream = bf16(400, HIDDEN), torch.empty_like(before), before.clone()
    x[24:] = float("nan")
    rows = 24 + long + 76
    caches = [[t.clone() for t in c] for c in layer.caches]
    step, ids = requests.step(_on([19, 5, long, 200]), rows)
    layer.attended.fill_(float("nan"))
    layer.normed(x[:rows], **step, max_queries=300, residual=stream[:rows], weight=weight, out=out[:rows], ids=ids)
    assert requests.granted.tolist() == [19, 5, 0, 0] and requests.q_starts.tolist() == [0, 19, 24, 24 + long, rows]
    assert step["lengths"].tolist() == [19, 5, 0, 0] and requests.pages.lengths.tolist() == [19, 5, 0, 0]
    assert (step["slots"][24:] == -1).all() and (ids[24:] == -1).all()
    _check_caches(layer, caches, x[:rows], [(0, 24, step["slots"][:24].cpu())])
    assert not layer.attended[:, 24:rows].any() and torch.equal(stream[24:], before[24:])
    assert stream.isfinite().all() and out[:rows].isfinite().all() and not torch.equal(stream[:24], before[:24])
