"""Rows of a step that are no sequence's: the serving layer adds nothing for them, whatever its buffers and the rows hold."""
import pytest
import torch

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
